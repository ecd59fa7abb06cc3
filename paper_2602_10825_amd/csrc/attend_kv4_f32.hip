// Chunk-causal attention of fp32 queries on a clean region in 4 bits (kv4.hpp) and the active chunks' fp32 slots.  Products on
// the bf16 matrix cores, floats in three bf16 parts (f32_split.hpp).  A value of the 4-bit rows has two significant
// bits and is its own first part, so a product with it takes three of the six: a clean key costs half of
// what it costs attend_f32.hip's blocks, which also read 16 times its bytes.
//
// 32 query rows per block; its 8 wavefronts take every 8th 32-key tile of the range, as in attend_kv4.hip (FcAttendArgs
// describes the slots alone, the clean region's tiles come first).  Q's parts are in LDS for all wavefronts.  K's codes go straight
// into the product's operand, V's become bf16 rows in LDS that a transposing read turns; a slot's V is taken 32 columns at a time,
// its parts side by side in the same LDS.
// 12 x 128, on codes and the chunk's own slot: 256 rows on 49201 keys 220 us (attend_f32.hip on the unpacked rows 372), 353 TFLOP/s
// where a third of a large bf16 product's rate is 394: the matrix cores; one row on 61201 keys 47 us (200); 10200 rows on 40800
// keys and two slots 15.8 ms (16.8).  There the slots take half of the time, bound by the vector instructions that split their
// rows, 700 of 900 per tile: 130 TFLOP/s (attend_f32.hip's 256-row blocks: 197).
//
// Operands are finite; a part is lost below 2^-110, so entries of Q (times the scale) and of the slots hold all their bits from
// 2^-100 on.
#include "attend_split.hpp"
#include "f32_split.hpp"
#include "kv4_tiles.hpp"

namespace {

constexpr int BK = 32;               // keys per tile
constexpr int NT = kSplitThreads;
// The exponents' reference is raised this far beyond the row maximum when that passes it (log2): weights are at most 1.
constexpr float kAhead = 4.0f;

template <int D>
struct Smem {
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
    Segments sg;
};

template <int D>
__global__ __launch_bounds__(NT) void attend_kv4_f32_kernel(FcAttendArgs a, FcAttendPlan p, float* parts, FcKv4 x) {
    constexpr int KS = D / 16;           // contraction steps of Q K^T
    constexpr int NB = D / 32;           // 32-wide blocks of the value dimension
    constexpr int QROW = Smem<D>::QROW, OROW = Smem<D>::OROW;
    __shared__ Smem<D> sm;
    Segments& sg = sm.sg;

    const uint32_t valid = valid_blocks(a);
    if (valid == 0u) return;
    const SplitItem it = split_item(a, p, valid, blockIdx.x);
    if (!it.ok) return;
    const int hk = it.h / (a.H_q / a.H_k);
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int l32 = lane & 31, hh = lane >> 5;
    const float c2 = a.scale * 1.4426950408889634f;   // fold log2(e): exp(x) = exp2(x*log2 e)

    if (tid == 0) list_segments(a, it.c, sg);
    if (tid < kUnitRows * (D / 8)) {
        const int row = tid / (D / 8), e = tid % (D / 8);
        int rc = it.tile * kUnitRows + row;
        if (rc > a.L_c - 1) rc = a.L_c - 1;
        const float* qp = (const float*)a.q + (((int64_t)it.r * a.L_c + rc) * a.H_q + it.h) * D + 8 * e;
        const f32x4_t v0 = *reinterpret_cast<const f32x4_t*>(qp) * c2, v1 = *reinterpret_cast<const f32x4_t*>(qp + 4) * c2;
        Split8 s;
        split_pair(s, 0, v0[0], v0[1]); split_pair(s, 1, v0[2], v0[3]);
        split_pair(s, 2, v1[0], v1[1]); split_pair(s, 3, v1[2], v1[3]);
        *reinterpret_cast<u32x4_native*>(sm.t.q[0] + row * QROW + 8 * e) = s.h;
        *reinterpret_cast<u32x4_native*>(sm.t.q[1] + row * QROW + 8 * e) = s.m;
        *reinterpret_cast<u32x4_native*>(sm.t.q[2] + row * QROW + 8 * e) = s.l;
    }
    __syncthreads();
    const int tiles4 = (x.L_clean + BK - 1) / BK;
    const int nt = tiles4 + __builtin_amdgcn_readfirstlane(sg.tile0[sg.n]);
    const int t_end = (int)((int64_t)nt * (it.s + 1) / it.S);
    const int t_end4 = t_end < tiles4 ? t_end : tiles4;
    int t = (int)((int64_t)nt * it.s / it.S) + wave;

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

// 32-row blocks for every recompute count; how many ranges the keys of a block are divided into.
FcAttendPlan plan_of(const FcAttendArgs& a, int L_clean, bool may_split) {
    FcAttendPlan p{};
    p.tiles = (a.L_c + kUnitRows - 1) / kUnitRows;
    const int64_t keys = (int64_t)L_clean + (int64_t)a.A * a.L_c;
    for (int R = 1; R <= a.A; ++R) {
        int S = 1;
        const int64_t units = (int64_t)R * a.H_q * p.tiles;
        fc_narrow_cost(units, (int)((keys + BK - 1) / BK), 14, may_split, &S);
        p.narrow[R - 1] = 1;
        fc_plan_add(p, R, units * S, units, S);
    }
    return p;
}

template <int D>
int launch(FcAttendArgs a, const FcKv4& x, hipStream_t s) {
    a.L_clean = 0;                    // the slots alone
    FcAttendPlan p = plan_of(a, x.L_clean, true);
    if (!fc_room_for_partials(a.ws, a.ws_bytes, p.parts, D)) p = plan_of(a, x.L_clean, false);
    attend_kv4_f32_kernel<D><<<p.grid, NT, 0, s>>>(a, p, (float*)a.ws, x);
    FC_LAUNCH_CHECK();
    return launch_merge4<float, D>(a, p, s);
}

}  // namespace

int fc_launch_attend_kv4_f32(const FcAttendArgs& a, const FcKv4& x, hipStream_t s) {
    if (a.d == 128) return launch<128>(a, x, s);
    if (a.d == 64) return launch<64>(a, x, s);
    return FC_UNSUPPORTED;
}
