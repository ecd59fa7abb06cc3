// Chunk-causal attention of fp32 queries on a clean region in 4 bits (kv4.hpp) and the active chunks' fp32 slots.  Products on
// the bf16 matrix cores, floats in three bf16 parts (f32_split.hpp).  A value of the 4-bit rows has two significant
// bits and is its own first part, so a product with it takes three of the six: a clean key costs half of
// what it costs attend_f32.hip, which also reads 16 times its bytes.  Bodies, plan and divisions of the keys as there.
// us, attend_f32.hip on the unpacked rows / here, three sets of inputs in turn (no cache is found in the Infinity Cache): 12 x 128, one
// row on 61201 keys 193 / 45, 256 rows on 49201 388 / 227, 600 on 5200 140 / 78, 10200 on 40800 keys and two slots 16630 / 12390; 24 x 128,
// 2 chunks of 4000 rows on 20000 keys 11020 / 7750, 4 of 2340 on their slots alone 3520 / 3450; 24 x 64, 2 of 2040 rows on 18360 keys and
// 5 slots 3180 / 2560.  The large ones run at 309 and 330 TFLOP/s counted as fp32; a third (codes) and a sixth (slots) of a large bf16
// product's rate on that card, mixed as their keys are, 340 and 366: matrix cores.
//
// What has no parts or loses them (infinities, entries near the largest float, very small ones) is looked for in Q and in the sums, and
// the wavefront's rows are then formed again with fp32 products.
#include <type_traits>

#include "attend_split.hpp"
#include "f32_split.hpp"
#include "kv4_tiles.hpp"

namespace {

constexpr int BK = 32;               // keys per tile
constexpr int NT = kSplitThreads;
// The exponents' reference is raised this far beyond the row maximum when that passes it (log2): weights are at most 1.
constexpr float kAhead = 4.0f;

// Is there a sum of products of which parts were lost, or one that is infinite or not a number (then their total is too), or were there
// such rows of Q (`odd`)?  What a value or a weight loses is at most 2^-134 (half of bf16's least step), so a sum over all keys loses at
// most 2^-134 times the sum of weights: less than 2^-24 of it from 2^-110 times that sum on.  Zeros lost nothing.  (A key that
// outweighs all others by 76 in natural units and has zeros among its codes leaves such sums too; with a border of 2^-90 and the
// sums of weights looked at as well it was 62: 256 rows on 8000 keys, 16 of them 70 above the others, 63 us, and 160 then.
// 8 on 2 x 128, 328 rows on 1311 keys: nothing looked at 35.2 us, each sum compared by itself 36.2, this 35.9.)
template <int NB>
__device__ __forceinline__ bool again_in_fp32(bool odd, const f32x16_t (&o)[NB], float l) {
    auto rank = [](float x) { return (__float_as_uint(x) << 1) - 1u; };         // by magnitude, zero last
    float total = fabsf(l);
    uint32_t least = ~0u;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            total += fabsf(o[b][i]);
            least = rank(o[b][i]) < least ? rank(o[b][i]) : least;
        }
    const float weights = l + __shfl_xor(l, 32, FC_WAVE);
    return (__ballot(odd || least < rank(weights * 0x1p-110f)) | odd_sum(total)) != 0;
}

// The 32 rows of a wavefront over its tiles t, t + step, ... < t_end once more, with fp32 products.  `q` is the lane's own row from
// column 4 hh on; value column 32 b + l32 is row l32 of block b.  Slow: every wavefront reads its operands from memory.
template <int D>
__device__ __forceinline__ void rows_in_fp32(const float* q, const FcCodesHead& head, const float* kbase, const float* vbase, uint32_t ts,
                                             const Segments& sg, int t, int t_end, int step, float c2, int lane, f32x16_t (&o)[D / 32], float& m, float& l) {
    constexpr int NB = D / 32;
    const int l32 = lane & 31, hh = lane >> 5;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
    m = kNegBig;
    l = 0.f;
    f32x16_t s;
    auto scores = [&](int j, const f32x4_t& kf) __attribute__((always_inline)) {   // contracts over elements 8 j + i and 8 j + 4 + i
        const f32x4_t qf = *reinterpret_cast<const f32x4_t*>(q + 8 * j) * c2;
#pragma unroll
        for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[i], qf[i], s, 0, 0, 0);
    };
    auto weights = [&](int nv) __attribute__((always_inline)) {
        if (nv < BK) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if ((i >> 2) * 8 + hh * 4 + (i & 3) >= nv) s[i] = kNegBig;
        }
        float mx = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
        const float mn = fmaxf(m, fmaxf(mx, __shfl_xor(mx, 32, FC_WAVE))), alpha = __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        float ps = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) { s[i] = __builtin_amdgcn_exp2f(s[i] - mn); ps += s[i]; }
        l = fmaf(l, alpha, ps);
#pragma unroll
        for (int b = 0; b < NB; ++b) o[b] *= alpha;
    };
    // (keys past the end have the last one's value, which may be infinite, and no weight: zero instead)
    auto key_of = [&](int i) { return (i >> 2) * 8 + hh * 4 + (i & 3); };
    auto inside = [&](int i, int nv) { return (uint32_t)(key_of(i) < nv ? key_of(i) : nv - 1); };
    int seg = 0;
#pragma unroll 1
    for (; t < t_end; t += step) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
        if (t < head.tiles) {
            const int left = head.L_clean - t * BK, nv = left < BK ? left : BK;
            const uint8_t *kt = head.k + (int64_t)t * (16 * D), *vt = head.v + (int64_t)t * (16 * D);
            const uint8_t *kst = head.k + head.to_scales + (int64_t)t * D, *vst = head.v + head.to_scales + (int64_t)t * D;
            const uint32_t row = (uint32_t)(l32 < nv ? l32 : nv - 1);
#pragma unroll 2
            for (int j = 0; j < D / 8; ++j)
                scores(j, fc_kv4_to_f32(*reinterpret_cast<const uint16_t*>(kt + (row * (D / 2) + 4 * j + 2 * hh)), kst[row * (D / 32) + (j >> 2)]));
            weights(nv);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t key = inside(i, nv);
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const uint32_t two = vt[key * (D / 2) + 16 * b + (l32 >> 1)];
                    const f32x4_t v = fc_kv4_to_f32(l32 & 1 ? two >> 4 : two, vst[key * (D / 32) + b]);
                    o[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(key_of(i) < nv ? v[0] : 0.f, s[i], o[b], 0, 0, 0);
                }
                __builtin_amdgcn_sched_barrier(0);         // (few values in registers at a time)
            }
        } else {
            const int tt = t - head.tiles;
            while (tt >= __builtin_amdgcn_readfirstlane(sg.tile0[seg + 1])) ++seg;
            const int off = (tt - __builtin_amdgcn_readfirstlane(sg.tile0[seg])) * BK;
            const int left = __builtin_amdgcn_readfirstlane(sg.len[seg]) - off, nv = left < BK ? left : BK;
            const int64_t pos = (int64_t)(__builtin_amdgcn_readfirstlane(sg.start[seg]) + off) * ts;
            const float *kr = kbase + pos + (uint32_t)(l32 < nv ? l32 : nv - 1) * ts + 4 * hh, *vt = vbase + pos + l32;
#pragma unroll 2
            for (int j = 0; j < D / 8; ++j) scores(j, *reinterpret_cast<const f32x4_t*>(kr + 8 * j));
            weights(nv);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float* vr = vt + inside(i, nv) * ts;
#pragma unroll
                for (int b = 0; b < NB; ++b) o[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(key_of(i) < nv ? vr[32 * b] : 0.f, s[i], o[b], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
}

// ---- few query rows ---------------------------------------------------------------------
// 32 query rows per block; its 8 wavefronts take every 8th 32-key tile of the range, as in attend_kv4.hip (FcAttendArgs
// describes the slots alone, the clean region's tiles come first).  Q's parts are in LDS for all wavefronts.  K's codes go straight
// into the product's operand, V's become bf16 rows in LDS that a transposing read turns; a slot's V is taken 32 columns at a time,
// its parts side by side in the same LDS.  On codes 353 TFLOP/s of those 394; a slot's tile takes three times as long, 40 % of it waiting
// for its rows, which are too many to have two on their way.  Tried there: rows read in whole lines (the same), residues of
// the splitting by products of pairs instead of shifts (a third fewer vector instructions, the same).
template <int D>
struct NarrowSmem {
    static constexpr int QROW = D + 8, OROW = D + 4;
    static constexpr int TILE = 32 * (D > 3 * 32 ? D : 3 * 32);      // a tile of codes, or 32 columns of a slot's in three parts
    __attribute__((aligned(16))) union {
        struct {
            bf16_t q[3][kUnitRows * QROW];              // Q's parts: first, or their addresses take a register each
            bf16_t v[kSplitWaves][TILE];                // one tile per wavefront
        } t;
        float o[kSplitWaves * kUnitRows * OROW];        // partial O at the end
    };
    float m_s[kSplitWaves * kUnitRows], l_s[kSplitWaves * kUnitRows];
    __attribute__((aligned(16))) uint32_t odd[kSplitWaves];   // rows of Q that need fp32 products, by the wavefront that split them
    Segments sg;
};

template <int D>
__device__ __forceinline__ void attend_narrow(const FcAttendArgs& a, const FcAttendPlan& p, uint32_t valid, NarrowSmem<D>& sm,
                                              float* parts, const FcKv4& x) {
    constexpr int KS = D / 16;           // contraction steps of Q K^T
    constexpr int NB = D / 32;           // 32-wide blocks of the value dimension
    constexpr int QROW = NarrowSmem<D>::QROW, OROW = NarrowSmem<D>::OROW;
    Segments& sg = sm.sg;

    const SplitItem it = split_item(a, p, valid, blockIdx.x);
    if (!it.ok) return;
    const int hk = it.h / (a.H_q / a.H_k);
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int l32 = lane & 31, hh = lane >> 5;
    const float c2 = a.scale * 1.4426950408889634f;   // fold log2(e): exp(x) = exp2(x*log2 e)

    auto q_row = [&](int row) {
        int rc = it.tile * kUnitRows + row;
        if (rc > a.L_c - 1) rc = a.L_c - 1;
        return (const float*)a.q + (((int64_t)it.r * a.L_c + rc) * a.H_q + it.h) * D;
    };

    if (tid == 0) list_segments(a, it.c, sg);
    bool odd = false;
    if (tid < kUnitRows * (D / 8)) {
        const int row = tid / (D / 8), e = tid % (D / 8);
        const float* qp = q_row(row) + 8 * e;
        const f32x4_t v0 = *reinterpret_cast<const f32x4_t*>(qp) * c2, v1 = *reinterpret_cast<const f32x4_t*>(qp + 4) * c2;
#pragma unroll
        for (int i = 0; i < 4; ++i) odd |= odd_magnitude(v0[i]) | odd_magnitude(v1[i]);
        Split8 s;
        split_pair(s, 0, v0[0], v0[1]); split_pair(s, 1, v0[2], v0[3]);
        split_pair(s, 2, v1[0], v1[1]); split_pair(s, 3, v1[2], v1[3]);
        *reinterpret_cast<u32x4_native*>(sm.t.q[0] + row * QROW + 8 * e) = s.h;
        *reinterpret_cast<u32x4_native*>(sm.t.q[1] + row * QROW + 8 * e) = s.m;
        *reinterpret_cast<u32x4_native*>(sm.t.q[2] + row * QROW + 8 * e) = s.l;
    }
    odd = __any(odd);
    if (lane == 0) sm.odd[wave] = odd;
    __syncthreads();
    const int tiles4 = (x.L_clean + BK - 1) / BK;
    const int nt = tiles4 + __builtin_amdgcn_readfirstlane(sg.tile0[sg.n]);
    const int t_end = (int)((int64_t)nt * (it.s + 1) / it.S);
    const int t_end4 = t_end < tiles4 ? t_end : tiles4;
    const int t_first = (int)((int64_t)nt * it.s / it.S) + wave;
    int t = t_first;

    f32x16_t o[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
    float m = kNegBig, l = 0.f;
    bf16_t* vw = sm.t.v[wave];

    // B operand of S^T = K Q^T: lane has Q[q = l32][hh D / 2 + 8 step .. + 8)
    const int q_frag = l32 * QROW + hh * (D / 2);
    auto read_q = [&](int st) {
        return Split8{*reinterpret_cast<const u32x4_native*>(&sm.t.q[0][q_frag + 8 * st]),
                      *reinterpret_cast<const u32x4_native*>(&sm.t.q[1][q_frag + 8 * st]),
                      *reinterpret_cast<const u32x4_native*>(&sm.t.q[2][q_frag + 8 * st])};
    };
    auto zero = [&](f32x16_t& y) {
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = 0.f;
    };
    // scores of a tile -> its weights in parts, m, l, and O to the new reference
    auto weigh = [&](f32x16_t& s, int nv, Split8 (&ps)[2]) {
        if (nv < BK) {
            const int mine = nv - hh * 4;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if ((i >> 2) * 8 + (i & 3) >= mine) s[i] = kNegBig;
        }
        float mx = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
        if (__any(mx > m)) {
            const float top = fmaxf(mx, __shfl_xor(mx, 32, FC_WAVE)), mn = top > m ? top + kAhead : m;
            const float alpha = __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= alpha;
#pragma unroll
            for (int b = 0; b < NB; ++b) o[b] *= alpha;
        }
        float p0 = 0.f, p1 = 0.f;
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float x0 = __builtin_amdgcn_exp2f(s[i] - m), x1 = __builtin_amdgcn_exp2f(s[i + 1] - m);
            p0 += x0;
            p1 += x1;
            split_pair(ps[i >> 3], (i & 7) >> 1, x0, x1);
        }
        l += p0 + p1;
    };
    const int l16 = lane & 15, v_row = hh * 4 + (l16 >> 2);
    auto read_v = [&](const bf16_t* lo_at, const bf16_t* hi_at) {
        const s16x4_t lo = lds_read_tr(lo_at), hi = lds_read_tr(hi_at);
        return __builtin_bit_cast(u32x4_native, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };

    // ---- tiles of codes: two on their way while a third is worked on
    if (t < t_end4) {
        const FcCodesHead head{x.k + (int64_t)hk * x.head_codes, x.v + (int64_t)hk * x.head_codes,
                               x.scales_at + (int64_t)hk * (x.head_scales - x.head_codes), x.L_clean, tiles4};
        const int v_at = v_row * D + fc_swapped<D>(v_row, ((lane >> 4) & 1) * 2 + ((l16 & 3) >> 1)) * 8 + (l16 & 1) * 4;
        const int st_row = l32 * D, st_swap = fc_swapped<D>(l32, hh * (D / 16)) * 8;
        auto codes_tile = [&](FcCodes<D>& c, int tt) {
            f32x16_t s, s1;                                // the products with Q's first parts, and the others
            zero(s); zero(s1);
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                const u32x4_native kf = c.key(st);
                const Split8 q = read_q(st);
                split_mfma(kf, q.l, s1);
                split_mfma(kf, q.m, s1);
                split_mfma(kf, q.h, s);
            }
            s += s1;
            // the wavefront's own tile: its LDS accesses are served in order, no barrier is needed
#pragma unroll
            for (int st = 0; st < KS; ++st) *reinterpret_cast<u32x4_native*>(&vw[st_row + (st_swap ^ (st * 8))]) = c.value(st);
            const int nv = x.L_clean - tt * BK < BK ? x.L_clean - tt * BK : BK;
            c.fetch(head, tt + 2 * kSplitWaves, l32, hh);
            Split8 ps[2];
            weigh(s, nv, ps);
#pragma unroll
            for (int tt2 = 0; tt2 < 2; ++tt2)
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const u32x4_native vf = read_v(vw + ((v_at ^ (b * 32)) + tt2 * 16 * D), vw + ((v_at ^ (b * 32) ^ 8) + (tt2 * 16 + 8) * D));
                    split_mfma(vf, ps[tt2].l, o[b]);
                    split_mfma(vf, ps[tt2].m, o[b]);
                    split_mfma(vf, ps[tt2].h, o[b]);
                }
        };
        FcCodes<D> c0, c1;
        c0.fetch(head, t, l32, hh);
        c1.fetch(head, t + kSplitWaves, l32, hh);
        for (;;) {
            codes_tile(c0, t);
            t += kSplitWaves;
            if (t >= t_end4) break;
            codes_tile(c1, t);
            t += kSplitWaves;
            if (t >= t_end4) break;
        }
    }

    // ---- tiles of the slots' rows: a lane has half of K's row l32, and of V's 16 columns of a block at a time
    int seg = 0, nvalid = 0;
    const uint32_t ts = (uint32_t)a.tok_stride;
    int64_t pos = 0;
    auto locate = [&](int tt) {
        tt -= tiles4;
        while (tt >= __builtin_amdgcn_readfirstlane(sg.tile0[seg + 1])) ++seg;
        const int off = (tt - __builtin_amdgcn_readfirstlane(sg.tile0[seg])) * BK;
        const int left = __builtin_amdgcn_readfirstlane(sg.len[seg]) - off;
        pos = (int64_t)hk * a.head_stride + (int64_t)(__builtin_amdgcn_readfirstlane(sg.start[seg]) + off) * a.tok_stride;
        nvalid = left < BK ? left : BK;
    };
    f32x4_t kr[2 * KS];
    auto load_k = [&]() {
        const float* kt = (const float*)a.k_cache + pos;
        const uint32_t at = (uint32_t)(l32 < nvalid ? l32 : nvalid - 1) * ts + (uint32_t)(hh * (D / 2));   // rows past the end: the last one
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) kr[i] = *reinterpret_cast<const f32x4_t*>(kt + at + 4 * i);
    };
    if (t < t_end) { locate(t); load_k(); }
    while (t < t_end) {
        const int nv = nvalid;
        f32x4_t vr[4 * NB];
        const float* vt = (const float*)a.v_cache + pos;
        const uint32_t vat = (uint32_t)(l32 < nv ? l32 : nv - 1) * ts + (uint32_t)(hh * 16);
        auto load_v = [&](int b0, int b1) {
#pragma unroll
            for (int i = 4 * b0; i < 4 * b1; ++i) vr[i] = *reinterpret_cast<const f32x4_t*>(vt + vat + (i >> 2) * 32 + 4 * (i & 3));
        };
        load_v(0, NB / 2);
        f32x16_t s, s1;
        zero(s); zero(s1);
#pragma unroll
        for (int st = 0; st < KS; ++st) {
            Split8 k;
#pragma unroll
            for (int e = 0; e < 4; ++e) split_pair(k, e, kr[2 * st + (e >> 1)][2 * (e & 1)], kr[2 * st + (e >> 1)][2 * (e & 1) + 1]);
            const Split8 q = read_q(st);
            split_mfma(k.l, q.h, s1);
            split_mfma(k.h, q.l, s1);
            split_mfma(k.m, q.m, s1);
            split_mfma(k.m, q.h, s1);
            split_mfma(k.h, q.m, s1);
            split_mfma(k.h, q.h, s);
        }
        s += s1;
        load_v(NB / 2, NB);
        t += kSplitWaves;
        Split8 ps[2];
        weigh(s, nv, ps);
        // a part's block: rows of four 16-byte pieces, exchanged by the row's number in fours
        const int w_at = l32 * 32, w_swap = (l32 >> 2) & 3;
        const int r_at = v_row * 32 + (l16 & 1) * 4, r_piece = ((lane >> 4) & 1) * 2 + ((l16 & 3) >> 1);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {                  // 8 of the 16 columns
                Split8 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) split_pair(v, e, vr[4 * b + 2 * i + (e >> 1)][2 * (e & 1)], vr[4 * b + 2 * i + (e >> 1)][2 * (e & 1) + 1]);
                const int at = w_at + ((hh * 2 + i) ^ w_swap) * 8;
                *reinterpret_cast<u32x4_native*>(&vw[at]) = v.h;
                *reinterpret_cast<u32x4_native*>(&vw[32 * 32 + at]) = v.m;
                *reinterpret_cast<u32x4_native*>(&vw[2 * 32 * 32 + at]) = v.l;
            }
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
                const int lo = r_at + tt * 16 * 32 + (r_piece ^ hh) * 8, hi = r_at + (tt * 16 + 8) * 32 + (r_piece ^ hh ^ 2) * 8;
                const u32x4_native vh = read_v(vw + lo, vw + hi), vm = read_v(vw + 32 * 32 + lo, vw + 32 * 32 + hi);
                const u32x4_native vl = read_v(vw + 2 * 32 * 32 + lo, vw + 2 * 32 * 32 + hi);
                split_mfma(vl, ps[tt].h, o[b]);
                split_mfma(vh, ps[tt].l, o[b]);
                split_mfma(vm, ps[tt].m, o[b]);
                split_mfma(vm, ps[tt].h, o[b]);
                split_mfma(vh, ps[tt].m, o[b]);
                split_mfma(vh, ps[tt].h, o[b]);
            }
            if (b == NB / 2 - 1 && t < t_end) { locate(t); load_k(); }   // half of V is used up: its registers are free
        }
    }

    const u32x4_native odd0 = *reinterpret_cast<const u32x4_native*>(sm.odd), odd1 = *reinterpret_cast<const u32x4_native*>(sm.odd + 4);
    odd = (odd0[0] | odd0[1] | odd0[2] | odd0[3] | odd1[0] | odd1[1] | odd1[2] | odd1[3]) != 0u;
    if (__builtin_expect(again_in_fp32<NB>(odd, o, l), 0)) {
        const FcCodesHead head{x.k + (int64_t)hk * x.head_codes, x.v + (int64_t)hk * x.head_codes,
                               x.scales_at + (int64_t)hk * (x.head_scales - x.head_codes), x.L_clean, tiles4};
        rows_in_fp32<D>(q_row(l32) + 4 * hh, head, (const float*)a.k_cache + (int64_t)hk * a.head_stride,
                        (const float*)a.v_cache + (int64_t)hk * a.head_stride, ts, sg, t_first, t_end, kSplitWaves, c2, lane, o, m, l);
    }

    l += __shfl_xor(l, 32, FC_WAVE);
    __syncthreads();                                    // every wavefront is done with its tiles and with Q
    if (hh == 0) { sm.m_s[wave * kUnitRows + l32] = m; sm.l_s[wave * kUnitRows + l32] = l; }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4_t*>(&sm.o[(wave * kUnitRows + l32) * OROW + b * 32 + g * 8 + hh * 4]) =
                f32x4_t{o[b][4 * g], o[b][4 * g + 1], o[b][4 * g + 2], o[b][4 * g + 3]};
    __syncthreads();
    finish_unit<float, D, OROW>(a, p, it, sm.o, sm.m_s, sm.l_s, parts);
}

// ---- many query rows ----------------------------------------------------------------------------
// The 256-row body of attend_f32.hip: Q in registers, every 32-key tile read once, turned into parts once and double-buffered in
// LDS, a tile's contribution to O summed up by itself (added up in O directly: 11280 instead of 11830 us on 12 x 128, 10200 rows
// on 40800 keys, but a relative error of 24e-7 instead of 9e-7, which is attend_f32.hip's).  A tile of codes has one part
// and three products.  There is a loop for tiles of codes and one for slots' (at every step's choice between them the registers of both
// would be live), and one step that goes from the one to the other.
template <int D>
struct WideSmem {
    static constexpr int KROW = D + 8, VROW = D + 32;
    __attribute__((aligned(16))) bf16_t K[2][3][BK * KROW], V[2][3][BK * VROW];   // [buffer][part]; of codes the first part alone
    static constexpr int QL = D == 128 ? 6 : 0;      // steps of which Q's last part is kept here, every wavefront's own
    u32x4_native ql[QL > 0 ? QL : 1][kSplitWaves][FC_WAVE];
    Segments sg;
};

// The end of a block: sums that have to be formed again, then the result or the partial.  The thread's numbers are formed anew: kept
// through the loops for this, they take registers that the loops have not got (one of Q's operands was read back from memory in each
// tile, 12040 -> 12260 us on 12 x 128, 10200 rows on 40800 keys and two slots; now as without the look at the sums, within 0.3 %).
template <int D>
__device__ __forceinline__ void finish_wide(const FcAttendArgs& a, const FcAttendPlan& p, const WideItem& wi, const Segments& sg, int hk, int t_lo,
                                            int nt, int tiles4, float c2, bool odd, f32x16_t (&o)[D / 32], float m, float l, float* parts, const FcKv4& x4) {
    constexpr int NB = D / 32;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int row_in_chunk = wi.tile * kWideRows + wave * 32 + l32;
    const float* q_row = (const float*)a.q + (((int64_t)wi.r * a.L_c + (row_in_chunk > a.L_c - 1 ? a.L_c - 1 : row_in_chunk)) * a.H_q + wi.h) * D;
    if (__builtin_expect(again_in_fp32<NB>(odd, o, l), 0)) {
        const FcCodesHead head{x4.k + (int64_t)hk * x4.head_codes, x4.v + (int64_t)hk * x4.head_codes,
                               x4.scales_at + (int64_t)hk * (x4.head_scales - x4.head_codes), x4.L_clean, tiles4};
        rows_in_fp32<D>(q_row + 4 * hh, head, (const float*)a.k_cache + (int64_t)hk * a.head_stride, (const float*)a.v_cache + (int64_t)hk * a.head_stride,
                        (uint32_t)a.tok_stride, sg, t_lo, t_lo + nt, 1, c2, lane, o, m, l);
    }

    const float ltot = l + __shfl_xor(l, 32, FC_WAVE);
    if (wi.S > 1) {
        const int64_t part = (wi.unit * (kWideRows / kUnitRows) + wave) * wi.S + wi.s;   // 32 rows each
        float* po = parts + (part * kUnitRows + l32) * D;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                store_out(po + b * 32 + g * 8 + hh * 4, o[b][4 * g], o[b][4 * g + 1], o[b][4 * g + 2], o[b][4 * g + 3]);
        if (hh == 0) {
            float* ml = parts + (int64_t)p.parts * kUnitRows * D + part * 2 * kUnitRows;
            ml[l32] = m;
            ml[kUnitRows + l32] = ltot;
        }
        return;
    }
    if (row_in_chunk >= a.L_c) return;
    const float inv = 1.0f / ltot;
    const int64_t row = (int64_t)wi.r * a.L_c + row_in_chunk;
    float* op = (float*)a.out + (row * a.H_q + wi.h) * D;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            store_out(op + b * 32 + g * 8 + hh * 4, o[b][4 * g] * inv, o[b][4 * g + 1] * inv, o[b][4 * g + 2] * inv, o[b][4 * g + 3] * inv);
    if (a.lse && hh == 0)
        a.lse[(int64_t)wi.h * a.A * a.L_c + row] = (m + __builtin_amdgcn_logf(ltot)) * 0.6931471805599453f;
}

template <int D>
__device__ __forceinline__ void attend_wide(const FcAttendArgs& a, const FcAttendPlan& p, uint32_t valid, WideSmem<D>& sm,
                                            float* parts, const FcKv4& x4) {
    constexpr int KS = D / 16;           // contraction steps of Q K^T
    constexpr int NB = D / 32;           // 32-wide blocks of the value dimension
    constexpr int KROW = WideSmem<D>::KROW, VROW = WideSmem<D>::VROW, QL = WideSmem<D>::QL;
    constexpr int EPT = BK * D / NT;     // entries of K, and of V, per thread and tile: all of one row
    constexpr int LPR = D / EPT;         // threads per row
    typedef uint32_t word_t __attribute__((ext_vector_type(EPT / 2)));
    static_assert(EPT == 8 || EPT == 4, "a thread's codes are 4 bytes or 2");
    typedef std::conditional_t<EPT == 8, uint32_t, uint16_t> codes_t;
    Segments& sg = sm.sg;

    const WideItem wi = wide_item<true>(a, p, valid, blockIdx.x);
    if (!wi.ok) return;
    const int hk = wi.h / (a.H_q / a.H_k);
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int l32 = lane & 31, hh = lane >> 5, l16 = lane & 15;
    const float c2 = a.scale * 1.4426950408889634f;
    if (tid == 0) list_segments(a, a.rec_idx[wi.r], sg);

    // B operand of S^T = K Q^T: lane holds Q[q = l32][16 st + 8 hh .. + 8)
    const int row_in_chunk = wi.tile * kWideRows + wave * 32 + l32;
    const float* q_row = (const float*)a.q + (((int64_t)wi.r * a.L_c + (row_in_chunk > a.L_c - 1 ? a.L_c - 1 : row_in_chunk)) * a.H_q + wi.h) * D;
    Split8 qf[KS];
    // odd_magnitude() of an entry times c2, without that product (which the splitting forms with the differences that follow it)
    const float small = 0x1p-100f / c2, large = 0x1p100f / c2;
    auto odd_entry = [&](float x) __attribute__((always_inline)) { return x != 0.f && !(fabsf(x) >= small && fabsf(x) < large); };
    bool odd = false;
#pragma unroll
    for (int st = 0; st < KS; ++st) {
        const f32x4_t q0 = *reinterpret_cast<const f32x4_t*>(q_row + 16 * st + 8 * hh), q1 = *reinterpret_cast<const f32x4_t*>(q_row + 16 * st + 8 * hh + 4);
        const f32x4_t x0 = q0 * c2, x1 = q1 * c2;
#pragma unroll
        for (int i = 0; i < 4; ++i) odd = odd || odd_entry(q0[i]) || odd_entry(q1[i]);
        split_pair(qf[st], 0, x0[0], x0[1]); split_pair(qf[st], 1, x0[2], x0[3]);
        split_pair(qf[st], 2, x1[0], x1[1]); split_pair(qf[st], 3, x1[2], x1[3]);
        if (st < QL) sm.ql[st][wave][lane] = qf[st].l;
    }
    odd = __any(odd);
    __syncthreads();

    const int tiles4 = (x4.L_clean + BK - 1) / BK;
    const int nt_all = tiles4 + __builtin_amdgcn_readfirstlane(sg.tile0[sg.n]);
    const int t_lo = (int)((int64_t)nt_all * wi.s / wi.S), nt = (int)((int64_t)nt_all * (wi.s + 1) / wi.S) - t_lo;
    const int n_codes = tiles4 - t_lo < 0 ? 0 : tiles4 - t_lo < nt ? tiles4 - t_lo : nt;    // the range's first tiles

    f32x16_t o[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
    float m = kNegBig, l = 0.f;

    // tile t of the range -> registers, entries of one row per thread; rows past the end: the last one again
    const int ld_row = tid / LPR, ld_col = EPT * (tid % LPR);
    int nv_load = BK;                                 // valid keys of the tile loaded last
    uint32_t kc = 0, vc = 0, ks = 0, vs = 0;
    auto load_codes = [&](int t) __attribute__((always_inline)) {
        const int tt = t_lo + t, left = x4.L_clean - tt * BK;
        nv_load = left < BK ? left : BK;
        const uint32_t row = (uint32_t)(ld_row < nv_load ? ld_row : nv_load - 1);
        const int64_t codes = (int64_t)hk * x4.head_codes + (int64_t)tt * (BK * D / 2), scales = x4.scales_at + (int64_t)hk * x4.head_scales + (int64_t)tt * D;
        const uint32_t at = row * (D / 2) + ld_col / 2, s_at = row * (D / 32) + ld_col / 32;
        kc = *reinterpret_cast<const codes_t*>(x4.k + codes + at);
        vc = *reinterpret_cast<const codes_t*>(x4.v + codes + at);
        ks = *(x4.k + scales + s_at);
        vs = *(x4.v + scales + s_at);
    };
    f32x4_t kr[EPT / 4], vr[EPT / 4];
    const float* kbase = (const float*)a.k_cache + (int64_t)hk * a.head_stride;
    const float* vbase = (const float*)a.v_cache + (int64_t)hk * a.head_stride;
    const uint32_t ts = (uint32_t)a.tok_stride;
    int seg = 0;
    auto load_rows = [&](int t) __attribute__((always_inline)) {
        const int tt = t_lo + t - tiles4;
        while (tt >= __builtin_amdgcn_readfirstlane(sg.tile0[seg + 1])) ++seg;
        const int off = (tt - __builtin_amdgcn_readfirstlane(sg.tile0[seg])) * BK;
        const int left = __builtin_amdgcn_readfirstlane(sg.len[seg]) - off;
        const int64_t pos = (int64_t)(__builtin_amdgcn_readfirstlane(sg.start[seg]) + off) * a.tok_stride;
        nv_load = left < BK ? left : BK;
        const uint32_t at = (uint32_t)(ld_row < nv_load ? ld_row : nv_load - 1) * ts + (uint32_t)ld_col;
#pragma unroll
        for (int j = 0; j < EPT / 4; ++j) {
            kr[j] = *reinterpret_cast<const f32x4_t*>(kbase + pos + at + 4 * j);
            vr[j] = *reinterpret_cast<const f32x4_t*>(vbase + pos + at + 4 * j);
        }
    };
    // What lies beyond the 16 bits of an access's own offset is reached from addresses that the compiler takes as given (or it
    // keeps one register for each access).
    auto given = [&](auto* at) __attribute__((always_inline)) {
        uint32_t off = (uint32_t)(reinterpret_cast<char*>(at) - reinterpret_cast<char*>(&sm));
        asm("" : "+v"(off));
        return reinterpret_cast<decltype(at)>(reinterpret_cast<char*>(&sm) + off);
    };
    bf16_t* const v_st = given(&sm.V[0][0][ld_row * VROW + ld_col]);
    const u32x4_native* const ql_at = given(&sm.ql[0][wave][lane]);
    const int st_k = ld_row * KROW + ld_col;
    auto store_part = [&](bf16_t* at, const u32x4_native& x) __attribute__((always_inline)) {
        word_t w;
#pragma unroll
        for (int i = 0; i < EPT / 2; ++i) w[i] = x[i];
        *reinterpret_cast<word_t*>(at) = w;
    };
    // The loaded tile into buffer `buf`, in KS pieces: codes in the first two, of rows a pair of K's or V's entries each.
    Split8 sp;
    auto stage = [&](auto codes, int buf, int e) __attribute__((always_inline)) {
        if constexpr (decltype(codes)::value) {
            if (e == 0) store_part(&sm.K[buf][0][st_k], fc_kv4_to_bf16(kc, ks));
            if (e == 1) store_part(v_st + buf * (3 * BK * VROW), fc_kv4_to_bf16(vc, vs));
        } else {
            const bool v = e >= EPT / 2;
            const int i = v ? e - EPT / 2 : e;
            const f32x4_t& f = v ? vr[i >> 1] : kr[i >> 1];
            split_pair(sp, i, f[2 * (i & 1)], f[2 * (i & 1) + 1]);
            if (i < EPT / 2 - 1) return;
#pragma unroll
            for (int part = 0; part < 3; ++part)
                store_part(v ? v_st + (buf * 3 + part) * (BK * VROW) : &sm.K[buf][part][st_k], part == 0 ? sp.h : part == 1 ? sp.m : sp.l);
        }
    };
    const int k_frag = l32 * KROW + 8 * hh;
    const bf16_t* const v_at = given(&sm.V[0][0][(hh * 4 + (l16 >> 2)) * VROW + ((lane >> 4) & 1) * 16 + (l16 & 3) * 4]);
    auto read_k = [&](int buf, int part, int st) __attribute__((always_inline)) {
        return *reinterpret_cast<const u32x4_native*>(&sm.K[buf][part][k_frag + 16 * st]);
    };
    auto read_v = [&](int buf, int part, int g) __attribute__((always_inline)) {    // g: value block g / 2, 16-key step g % 2
        const bf16_t* vp = v_at + ((buf * 3 + part) * (BK * VROW) + (g % 2) * 16 * VROW + (g / 2) * 32);
        const s16x4_t lo = lds_read_tr(vp), hi = lds_read_tr(vp + 8 * VROW);
        return __builtin_bit_cast(u32x4_native, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };

    int nv = 0;
    // Tile t, which is one of codes or not, as tile t + 1 is
    auto step = [&](auto codes, auto next_codes, int t) __attribute__((always_inline)) {
        constexpr bool C = decltype(codes)::value;
        const int buf = t & 1;
        f32x16_t s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
        auto q_last = [&](int st) __attribute__((always_inline)) { return st < QL ? ql_at[st * (kSplitWaves * FC_WAVE)] : qf[st].l; };
        // the smaller products first: then only the largest ones, K's first parts read once more, round the scores' bits
        __builtin_amdgcn_s_setprio(1);
        if constexpr (C) {
            u32x4_native f0 = read_k(buf, 0, 0), f1;
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                f1 = read_k(buf, 0, (st + 1) % KS);
                const u32x4_native ql = q_last(st);
                split_mfma(f0, ql, s);
                __builtin_amdgcn_sched_barrier(0);
                stage(next_codes, buf ^ 1, st);
                split_mfma(f0, qf[st].m, s);
                __builtin_amdgcn_sched_barrier(0);
                f0 = f1;
            }
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                if (st + 1 < KS) f1 = read_k(buf, 0, st + 1);
                split_mfma(f0, qf[st].h, s);
                __builtin_amdgcn_sched_barrier(0);
                f0 = f1;
            }
        } else {
            Split8 f0 = {read_k(buf, 0, 0), read_k(buf, 1, 0), read_k(buf, 2, 0)}, f1;
            u32x4_native h0, h1, h2;
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                if (st + 1 < KS) f1 = Split8{read_k(buf, 0, st + 1), read_k(buf, 1, st + 1), read_k(buf, 2, st + 1)};
                else { h0 = read_k(buf, 0, 0); h1 = read_k(buf, 0, 1); }
                const u32x4_native ql = q_last(st);
                split_mfma(f0.l, qf[st].h, s);
                split_mfma(f0.m, qf[st].m, s);
                __builtin_amdgcn_sched_barrier(0);
                stage(next_codes, buf ^ 1, st);
                split_mfma(f0.m, qf[st].h, s);
                split_mfma(f0.h, ql, s);
                split_mfma(f0.h, qf[st].m, s);
                __builtin_amdgcn_sched_barrier(0);
                f0 = f1;
            }
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                if (st + 2 < KS) h2 = read_k(buf, 0, st + 2);
                split_mfma(h0, qf[st].h, s);
                __builtin_amdgcn_sched_barrier(0);
                h0 = h1;
                h1 = h2;
            }
        }
        __builtin_amdgcn_s_setprio(0);
        auto read_parts = [&](int g) __attribute__((always_inline)) {
            if constexpr (C) return read_v(buf, 0, g);
            else return Split8{read_v(buf, 0, g), read_v(buf, 1, g), read_v(buf, 2, g)};
        };
        auto va = read_parts(0), na = va;
        if (nv < BK) {
            const int mine = nv - hh * 4;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if ((i >> 2) * 8 + (i & 3) >= mine) s[i] = kNegBig;
        }
        nv = nv_load;                                  // of tile t + 1
        float mx = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
        if (__any(mx > m)) {
            const float top = fmaxf(mx, __shfl_xor(mx, 32, FC_WAVE)), mn = top > m ? top + kAhead : m;
            const float alpha = __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= alpha;
#pragma unroll
            for (int b = 0; b < NB; ++b) o[b] *= alpha;
        }
        float p0 = 0.f, p1 = 0.f;
        Split8 ps[2];
        auto weights = [&](int i) __attribute__((always_inline)) {      // of accumulators i and i + 1
            const float x0 = __builtin_amdgcn_exp2f(s[i] - m), x1 = __builtin_amdgcn_exp2f(s[i + 1] - m);
            p0 += x0;
            p1 += x1;
            split_pair(ps[i >> 3], (i & 7) >> 1, x0, x1);
        };
#pragma unroll
        for (int i = 0; i < 8; i += 2) weights(i);
        f32x16_t x;
#pragma unroll
        for (int g = 0; g < 2 * NB; ++g) {                 // value block g / 2, 16-key step g % 2
            if (g % 2 == 0) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = 0.f;
            }
            if (g + 1 < 2 * NB) na = read_parts(g + 1);
            const Split8& pc = ps[g % 2];
            if constexpr (C) {
                split_mfma(va, pc.l, x); if (g == 0) { weights(8); weights(10); } __builtin_amdgcn_sched_barrier(0);
                split_mfma(va, pc.m, x); if (g == 0) { weights(12); weights(14); } __builtin_amdgcn_sched_barrier(0);
                split_mfma(va, pc.h, x);
            } else {
                split_mfma(va.l, pc.h, x); if (g == 0) weights(8); __builtin_amdgcn_sched_barrier(0);
                split_mfma(va.h, pc.l, x); if (g == 0) weights(10); __builtin_amdgcn_sched_barrier(0);
                split_mfma(va.m, pc.m, x); if (g == 0) weights(12); __builtin_amdgcn_sched_barrier(0);
                split_mfma(va.m, pc.h, x); if (g == 0) weights(14); __builtin_amdgcn_sched_barrier(0);
                split_mfma(va.h, pc.m, x); __builtin_amdgcn_sched_barrier(0);
                split_mfma(va.h, pc.h, x);
            }
            va = na;
            if (g % 2 == 1) o[g / 2] += x;
            if (g == 1 && t + 2 < nt) {                    // (the scores' registers are free)
                if (decltype(next_codes)::value && t + 2 < n_codes) load_codes(t + 2);
                else load_rows(t + 2);
            }
        }
        l += p0 + p1;
        lds_barrier();
    };
    if (nt > 0) {
        const std::true_type codes;
        const std::false_type rows;
        if (n_codes > 0) {
            load_codes(0);
            nv = nv_load;
#pragma unroll
            for (int e = 0; e < KS; ++e) stage(codes, 0, e);
        } else {
            load_rows(0);
            nv = nv_load;
#pragma unroll
            for (int e = 0; e < KS; ++e) stage(rows, 0, e);
        }
        if (nt > 1) {
            if (n_codes > 1) load_codes(1);
            else load_rows(1);
        }
        lds_barrier();
        int t = 0;
        const int whole = n_codes < nt ? n_codes - 1 : nt;         // tiles of codes before another (or nothing)
#pragma unroll 1
        for (; t < whole; ++t) step(codes, codes, t);
        if (t < n_codes) { step(codes, rows, t); ++t; }
#pragma unroll 1
        for (; t < nt; ++t) step(rows, rows, t);
    }

    finish_wide<D>(a, p, wi, sg, hk, t_lo, nt, tiles4, c2, odd, o, m, l, parts, x4);
}

// WIDE and NARROW say which of the two bodies some recompute count of this launch asks for.
template <int D, bool WIDE, bool NARROW>
__global__ __launch_bounds__(NT) void attend_kv4_f32_kernel(FcAttendArgs a, FcAttendPlan p, float* parts, FcKv4 x) {
    const uint32_t valid = valid_blocks(a);
    const int R = __popc(valid);
    if (R == 0) return;
    constexpr size_t w = WIDE ? sizeof(WideSmem<D>) : 0, n = NARROW ? sizeof(NarrowSmem<D>) : 0;
    __shared__ __attribute__((aligned(16))) char raw[w > n ? w : n];
    if (WIDE && (!NARROW || !p.narrow[R - 1]))
        attend_wide<D>(a, p, valid, *reinterpret_cast<WideSmem<D>*>(raw), parts, x);
    else if (NARROW)
        attend_narrow<D>(a, p, valid, *reinterpret_cast<NarrowSmem<D>*>(raw), parts, x);
}

template <int D>
int launch(FcAttendArgs a, const FcKv4& x, hipStream_t s) {
    a.L_clean = 0;                    // the slots alone
    FcAttendPlan p = fc_attend_plan_kv4_f32(a.A, a.L_c, x.L_clean, a.H_q, D, true);
    if (!fc_room_for_partials(a.ws, a.ws_bytes, p.parts, D)) p = fc_attend_plan_kv4_f32(a.A, a.L_c, x.L_clean, a.H_q, D, false);
    bool wide = false, narrow = false;
    for (int R = 0; R < a.A; ++R) (p.narrow[R] ? narrow : wide) = true;
    if (!narrow)
        attend_kv4_f32_kernel<D, true, false><<<p.grid, NT, 0, s>>>(a, p, (float*)a.ws, x);
    else if (!wide)
        attend_kv4_f32_kernel<D, false, true><<<p.grid, NT, 0, s>>>(a, p, (float*)a.ws, x);
    else
        attend_kv4_f32_kernel<D, true, true><<<p.grid, NT, 0, s>>>(a, p, (float*)a.ws, x);
    FC_LAUNCH_CHECK();
    return launch_merge4<float, D>(a, p, s);
}

}  // namespace

int fc_launch_attend_kv4_f32(const FcAttendArgs& a, const FcKv4& x, hipStream_t s) {
    if (a.d == 128) return launch<128>(a, x, s);
    if (a.d == 64) return launch<64>(a, x, s);
    return FC_UNSUPPORTED;
}
