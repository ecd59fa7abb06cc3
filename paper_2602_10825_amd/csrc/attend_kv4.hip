// Chunk-causal attention on a clean region in 4 bits (kv4.hpp) and the active chunks' bf16 slots: softmax(q K^T scale) V as
// in attend_bf16.hip, with the same division of the work, bodies and numerics.  The values that codes stand for have
// two significant bits: as bf16 operands they are exact, so nothing is rounded that the bf16 kernel does not round.
//
// In these kernels FcAttendArgs describes the slots alone (its L_clean is 0); the clean region, x.L_clean rows of the 4-bit
// buffers, comes first in the order of the key tiles and never shares a tile with a slot.
#include "attend_bf16.hpp"
#include "kv4_tiles.hpp"

namespace {

// ---- 256 query rows per block ---------------------------------------------------------------
// The body of attend_bf16.hip: its products, its ring of four K and two V tiles of bf16 rows in LDS, its one barrier per step and
// its rare raise of the exponents' reference.  A tile of codes becomes bf16 on its way into LDS: a thread has CPT neighbouring
// codes of one row and their scale's byte, 16 or 8 conversions and 2 or 1 writes each for K and V.  That is 20 of the 190 vector
// instructions of a step, and 136 bytes are read per key instead of 512; matrix cores and vector ALU bound it as they
// do there.
template <int D>
__device__ __forceinline__ void attend_wide4(const FcAttendArgs& a, const FcAttendPlan& p, uint32_t valid, WideSmem<D>& sm,
                                             float* parts, const FcKv4& x) {
    constexpr int KS = D / 16;        // contraction steps of Q K^T
    constexpr int DVB = D / 32;       // 32-wide blocks of the value dimension
    constexpr int KROW = WideSmem<D>::KROW, VROW = WideSmem<D>::VROW;
    constexpr int VPR = D / 8;        // 16-byte vectors per K/V row
    constexpr int LD = BK * VPR / NT; // global loads per thread per tile of rows (K, and again V)
    constexpr int CPT = BK * D / NT;  // codes per thread per tile
    constexpr float kTooBig = 1.0995116e12f;  // 2^40: a row sum above this triggers a raise of m
    constexpr int NPV = 4 * DVB, NQK = 2 * KS, N = NPV + NQK;   // matrix products of a step: P V, Q K^T
    constexpr int PF = 4;             // fragments are read this many products ahead

    const WideItem wi = wide_item<false>(a, p, valid, blockIdx.x);
    if (!wi.ok) return;
    const int r = wi.r, h = wi.h, tile = wi.tile;
    const int c = a.rec_idx[r];
    const int hk = h / (a.H_q / a.H_k);

    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;   // wave: scalar
    const int l32 = lane & 31, hh = lane >> 5;

    // ---- Q fragments (B operand of S^T = K Q^T): lane holds Q[q = l32][16*step + 8*hh ..+8)
    bf16x8_t qf[KS];
    const int row_in_chunk = tile * BQ + wave * 32 + l32;
    {
        const int rc = row_in_chunk > a.L_c - 1 ? a.L_c - 1 : row_in_chunk;
        const bf16_t* qp = (const bf16_t*)a.q + (((int64_t)r * a.L_c + rc) * a.H_q + h) * D + 8 * hh;
#pragma unroll
        for (int st = 0; st < KS; ++st) qf[st] = *reinterpret_cast<const bf16x8_t*>(qp + 16 * st);
    }
    const float c2 = a.scale * 1.4426950408889634f;

    // ---- the slots' segments (adjacent ones merged) and this block's range of the 64-key tiles
    const int tiles4 = (x.L_clean + BK - 1) / BK;
    if (tid == 0) {
        int n = 0, i = 0, nt = tiles4;
        while (i <= c) {
            const int start = a.active_off[i];
            int len = a.L_c;
            ++i;
            while (i <= c && a.active_off[i] == start + len) { len += a.L_c; ++i; }
            sm.seg_start[n] = start; sm.seg_len[n] = len; ++n; nt += (len + BK - 1) / BK;
        }
        const int lo = (int)((int64_t)nt * wi.s / wi.S);
        int skip = lo - tiles4, sg = 0;
        while (sg < n - 1 && skip >= (sm.seg_len[sg] + BK - 1) / BK) { skip -= (sm.seg_len[sg] + BK - 1) / BK; ++sg; }
        sm.seg_first = lo < tiles4 ? -1 : sg;
        sm.off_first = lo < tiles4 ? lo * BK : skip * BK < sm.seg_len[sg] ? skip * BK : 0;
        sm.n_tiles = (int)((int64_t)nt * (wi.s + 1) / wi.S) - lo;
    }
    __syncthreads();
    const int nt = __builtin_amdgcn_readfirstlane(sm.n_tiles);
    int seg = __builtin_amdgcn_readfirstlane(sm.seg_first);       // -1: the clean region
    int start = 0, len = x.L_clean;
    if (seg >= 0) {
        start = __builtin_amdgcn_readfirstlane(sm.seg_start[seg]);
        len = __builtin_amdgcn_readfirstlane(sm.seg_len[seg]);
    }
    int t0 = __builtin_amdgcn_readfirstlane(sm.off_first);
    int to_step = nt - 1;             // tiles after the one (start, len, t0) point at
    // Of the range's tiles the first n4 are codes.  Steps before `whole4` store and load whole tiles of codes only (K runs three
    // tiles ahead); from n4 on nothing but rows.
    int n4 = seg < 0 ? (len - t0 + BK - 1) / BK : 0;
    n4 = n4 < nt ? n4 : nt;
    int whole4 = seg < 0 ? (len - t0) / BK : 0;
    whole4 = (whole4 < nt ? whole4 : nt) - 3;

    u32x4_native kreg[LD], vreg[LD];
    // (registers of their own: where both kinds of tile shared theirs, the compiler moved them behind the loads and waited for those)
    struct Codes { uint32_t w[CPT / 8], scale; } kcodes, vcodes;
    const int ld_row = tid / VPR, ld_col = tid % VPR;
    constexpr int RPP = NT / VPR;     // rows per pass of the block's loads
    const uint32_t ts = (uint32_t)a.tok_stride;
    const bf16_t* kbase = (const bf16_t*)a.k_cache + (int64_t)hk * a.head_stride;
    const bf16_t* vbase = (const bf16_t*)a.v_cache + (int64_t)hk * a.head_stride;
    const uint8_t *k4 = x.k + (int64_t)hk * x.head_codes, *v4 = x.v + (int64_t)hk * x.head_codes;
    const int64_t to_scales = x.scales_at + (int64_t)hk * (x.head_scales - x.head_codes);
    const int row4 = tid / (D / CPT), col4 = tid % (D / CPT) * CPT;

    // Tile -> registers: wavefront-uniform base plus a 32-bit byte offset per lane; rows past the end of a segment re-read its
    // last one.  K runs two tiles ahead of V.  pos: the tile's first row, of codes the row itself, else its element offset.
    int64_t pos_k, pos_v, pos_q0 = 0, pos_q1 = 0;
    int nv_k, nv_v, nv_q0 = BK, nv_q1 = BK;
    int in4_k, in4_v, in4_q0 = 0, in4_q1 = 0;
    auto advance = [&]() {            // to the next tile; the range's last one is loaded again and again
        if (to_step > 0) {
            --to_step;
            t0 += BK;
            if (t0 >= len) {
                ++seg;
                start = __builtin_amdgcn_readfirstlane(sm.seg_start[seg]);
                len = __builtin_amdgcn_readfirstlane(sm.seg_len[seg]);
                t0 = 0;
            }
        }
    };
    auto step_tile = [&]() {          // K's next tile; V's is the one K had two calls before
        pos_v = pos_q1; nv_v = nv_q1; in4_v = in4_q1;
        pos_q1 = pos_q0; nv_q1 = nv_q0; in4_q1 = in4_q0;
        in4_k = seg < 0;
        pos_k = (int64_t)(start + t0) * (in4_k ? 1 : a.tok_stride);
        nv_k = len - t0 < BK ? len - t0 : BK;
        pos_q0 = pos_k; nv_q0 = nv_k; in4_q0 = in4_k;
        advance();
    };
    uint32_t voff[LD];
#pragma unroll
    for (int i = 0; i < LD; ++i) voff[i] = ((uint32_t)(i * RPP + ld_row) * ts + (uint32_t)ld_col * 8u) * 2u;
    const uint32_t voff_row = ts * 2u;
    auto load_rows = [&](u32x4_native& dst, const bf16_t* base, int64_t pos, int nv, int i) {
        const char* b = reinterpret_cast<const char*>(base + pos);
        uint32_t off = voff[i];
        if (nv < BK) {
            const int over = i * RPP + ld_row - (nv - 1);
            off -= over > 0 ? (uint32_t)over * voff_row : 0u;
        }
        dst = *reinterpret_cast<const u32x4_native*>(b + off);
    };
    auto load_codes = [&](Codes& dst, const uint8_t* base, int64_t pos, int row) {
        const uint8_t* codes = base + pos * (D / 2);
        const uint8_t* scales = base + to_scales + pos * (D / 32);
        const uint32_t at = (uint32_t)(row * (D / 2) + col4 / 2);
        if constexpr (CPT == 16) {
            const uint2 w = *reinterpret_cast<const uint2*>(codes + at);
            dst.w[0] = w.x; dst.w[1] = w.y;
        } else {
            dst.w[0] = *reinterpret_cast<const uint32_t*>(codes + at);
        }
        dst.scale = scales[(uint32_t)(row * (D / 32) + col4 / 32)];
    };
    auto load_tile = [&](u32x4_native (&dst)[LD], Codes& dst4, const bf16_t* base, const uint8_t* base4, int in4, int64_t pos, int nv) {
        if (in4) {
            load_codes(dst4, base4, pos, row4 < nv ? row4 : nv - 1);
        } else {
#pragma unroll
            for (int i = 0; i < LD; ++i) load_rows(dst[i], base, pos, nv, i);
        }
    };
    auto store_codes = [&](bf16_t* to, const Codes& src) {
#pragma unroll
        for (int i = 0; i < CPT / 8; ++i) *reinterpret_cast<u32x4_native*>(to + 8 * i) = fc_kv4_to_bf16(src.w[i], src.scale);
    };
    const int st_k = ld_row * KROW + ld_col * 8, st_v = ld_row * VROW + ld_col * 8;
    const int st_k4 = row4 * KROW + col4, st_v4 = row4 * VROW + col4;
    auto store_k = [&](bf16_t* t, const u32x4_native (&src)[LD], const Codes& src4, int in4) {
        if (in4) {
            store_codes(t + st_k4, src4);
        } else {
#pragma unroll
            for (int i = 0; i < LD; ++i) *reinterpret_cast<u32x4_native*>(t + st_k + i * RPP * KROW) = src[i];
        }
    };
    // per-lane offsets of the fragment reads.  Transposing V read: lane s of a 16-lane group addresses
    // key (s/4), dv 4*(s%4) of the group's 4-key x 16-dv patch; groups 0/1 cover dv 0-15 / 16-31,
    // lane half = key half
    const int l16 = lane & 15;
    const int k_frag = l32 * KROW + 8 * hh;
    const int v_frag = (hh * 4 + (l16 >> 2)) * VROW + ((lane >> 4) & 1) * 16 + (l16 & 3) * 4;

    f32x16_t o[DVB], s[2];
#pragma unroll
    for (int dv = 0; dv < DVB; ++dv)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dv][i] = 0.f;
    float m = kNegBig, lsum = 0.f;
    u32x4_native P[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) P[t] = u32x4_native{0u, 0u, 0u, 0u};
    const bf16x2_t ones = {(__bf16)1.0f, (__bf16)1.0f};

    auto read_k = [&](const bf16_t* Kb, int f) {      // product f: key block f / KS, contraction step f % KS
        return *reinterpret_cast<const bf16x8_t*>(&Kb[(f / KS) * 32 * KROW + 16 * (f % KS)]);
    };
    auto read_v = [&](const bf16_t* Vb, int f) {      // product f: 16-key step f / DVB, value block f % DVB
        const bf16_t* vp = Vb + (f / DVB) * 16 * VROW + (f % DVB) * 32;
        const s16x4_t lo = lds_read_tr(vp), hi = lds_read_tr(vp + 8 * VROW);
        return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto mask_tail = [&](f32x16_t (&y)[2], int nv) {   // ragged end of a segment: keys past it
        // (the lane's part on one side, so that the other is a constant: 32 sums were kept in registers, and others spilled for it)
        const int mine = nv - hh * 4;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (kb * 32 + (i >> 2) * 8 + (i & 3) >= mine) y[kb][i] = kNegBig;
    };
    auto qk = [&](const bf16_t* Kb, f32x16_t (&y)[2]) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int i = 0; i < 16; ++i) y[kb][i] = 0.f;
#pragma unroll
            for (int st = 0; st < KS; ++st)
            {
                y[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_k(Kb, kb * KS + st), qf[st], y[kb], 0, 0, 0);
                if (st & 1) __builtin_amdgcn_sched_barrier(0);   // (few fragments in registers at a time)
            }
        }
    };
    float ps0, ps1;
    auto pack4 = [&](float x0, float x1, float x2, float x3, int q) {  // four weights: rounded to bf16, added to the row sum
        const bf16x2_t lo = {(__bf16)x0, (__bf16)x1}, hi = {(__bf16)x2, (__bf16)x3};
        uint32_t w0 = __builtin_bit_cast(uint32_t, lo), w1 = __builtin_bit_cast(uint32_t, hi);
        asm volatile("" : "+v"(w0), "+v"(w1));
        // the sums run over the ROUNDED weights, the ones V is multiplied with
        ps0 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w0), ones, ps0, false);
        ps1 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w1), ones, ps1, false);
        asm volatile("" : "+v"(ps0), "+v"(ps1));
        P[q >> 1][(q & 1) * 2] = w0;
        P[q >> 1][(q & 1) * 2 + 1] = w1;
    };

    if (nt > 0) {
        // ---- K(0), K(1) into the ring, K(2) and V(0) on their way, S(0); "V(-1)" finite (its P is zero)
        int nv_prev = BK, nv_cur, nv_next;   // valid keys of the tile before S's, of S's and of the next one
        {
            step_tile();
            nv_cur = nv_k;
            const int first4 = in4_k;
            load_tile(kreg, kcodes, kbase, k4, in4_k, pos_k, nv_k);
            step_tile();
            nv_next = nv_k;
            load_tile(vreg, vcodes, kbase, k4, in4_k, pos_k, nv_k);
            store_k(sm.K[0], kreg, kcodes, first4);
            store_k(sm.K[1], vreg, vcodes, in4_k);
            for (int i = tid; i < BK * VROW / 8; i += NT) reinterpret_cast<uint4*>(sm.V[1])[i] = make_uint4(0, 0, 0, 0);
            step_tile();
            load_tile(kreg, kcodes, kbase, k4, in4_k, pos_k, nv_k);
            load_tile(vreg, vcodes, vbase, v4, in4_v, pos_v, nv_v);
        }
        __syncthreads();
        qk(&sm.K[0][k_frag], s);
        if (nv_cur < BK) mask_tail(s, nv_cur);
        bf16x8_t frag[PF];
#pragma unroll
        for (int f = 0; f < PF; ++f) frag[f] = read_v(&sm.V[1][v_frag], f);
        float psum = 0.f;
        int j = 0;
        bool raise;
        // One step.  KIND says what the tiles are that it stores (K(j+2), V(j)) and loads (K(j+3), V(j+1)).
        constexpr int kRows = 0, kWhole4 = 1, kAny = 2;
        auto step = [&](auto KIND) __attribute__((always_inline)) {
            constexpr int kind = KIND;
            const bf16_t* Kn = &sm.K[(j + 1) & 3][k_frag];
            const bf16_t* Vp = &sm.V[(j + 1) & 1][v_frag];
            const bf16_t* Vn = &sm.V[j & 1][v_frag];
            bf16_t *Kw = sm.K[(j + 2) & 3], *Vw = sm.V[j & 1];
            const float mneg = -m;
            float wt[8];                               // weights on their way into P
            ps0 = ps1 = 0.f;
            constexpr int NEXP = NPV + KS - 1;         // products over which the exponentials are spread
            constexpr int BAR = NPV + KS / 2;
            __builtin_amdgcn_s_setprio(1);
            static_for<N>([&](auto F) __attribute__((always_inline)) {
                constexpr int f = F;
                // matrix cores: O += V P(j-1), then S(j+1) = K Q^T
                const bf16x8_t fr = frag[f % PF];
                if constexpr (f < NPV) {
                    o[f % DVB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr, __builtin_bit_cast(bf16x8_t, P[f / DVB]), o[f % DVB], 0, 0, 0);
                } else {
                    constexpr int g = f - NPV;
                    if constexpr (g % KS == 0) {
                        f32x16_t z;
#pragma unroll
                        for (int i = 0; i < 16; ++i) z[i] = 0.f;
                        s[g / KS] = z;
                    }
                    s[g / KS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr, qf[g % KS], s[g / KS], 0, 0, 0);
                }
                // LDS: the fragment of product f + PF
                if constexpr (f + PF < NPV) frag[f % PF] = read_v(Vp, f + PF);
                else if constexpr (f + PF < N) frag[f % PF] = read_k(Kn, f + PF - NPV);
                else frag[f % PF] = read_v(Vn, f + PF - N);
                // vector ALU: weights of tile j
                constexpr int e0 = f < NEXP ? 32 * f / NEXP : 32, e1 = f < NEXP ? 32 * (f + 1) / NEXP : 32;
                static_for<e1 - e0>([&](auto E) __attribute__((always_inline)) {
                    constexpr int e = e0 + E;
                    float w = __builtin_amdgcn_exp2f(fmaf(s[e >> 4][e & 15], c2, mneg));
                    asm volatile("" : "+v"(w));       // computed here, next to the matrix products
                    wt[e & 7] = w;
                });
                static_for<8>([&](auto Q) __attribute__((always_inline)) {
                    // weights q are ready, and the products with the P register they replace are issued
                    constexpr int q = Q, fe = ((q + 1) * 4 * NEXP + 31) / 32 - 1, fp = (q / 2 + 1) * DVB;
                    if constexpr (f == (fe > fp ? fe : fp))
                        pack4(wt[(4 * q) & 7], wt[(4 * q + 1) & 7], wt[(4 * q + 2) & 7], wt[(4 * q + 3) & 7], q);
                });
                // staging: K(j+2), V(j) to LDS, then the loads of K(j+3), V(j+1)
                if constexpr (kind == kRows) {
                    if constexpr (f >= 2 && f < 2 + LD)
                        *reinterpret_cast<u32x4_native*>(Kw + st_k + (f - 2) * RPP * KROW) = kreg[f - 2];
                    if constexpr (f >= 2 + LD && f < 2 + 2 * LD)
                        *reinterpret_cast<u32x4_native*>(Vw + st_v + (f - 2 - LD) * RPP * VROW) = vreg[f - 2 - LD];
                    if constexpr (f == 2 + 2 * LD) step_tile();
                    if constexpr (f >= 2 + 2 * LD && f < 2 + 3 * LD) {
                        load_rows(kreg[f - 2 - 2 * LD], kbase, pos_k, nv_k, f - 2 - 2 * LD);
                        load_rows(vreg[f - 2 - 2 * LD], vbase, pos_v, nv_v, f - 2 - 2 * LD);
                    }
                } else if constexpr (kind == kWhole4) {
                    if constexpr (f == 2) store_codes(Kw + st_k4, kcodes);
                    if constexpr (f == 3) store_codes(Vw + st_v4, vcodes);
                    // (what step_tile() does, where no tile is ragged and the next one follows)
                    if constexpr (f == 4) load_codes(kcodes, k4, t0, row4);
                    if constexpr (f == 5) {
                        load_codes(vcodes, v4, t0 - 2 * BK, row4);
                        t0 += BK;
                        --to_step;
                    }
                } else {
                    if constexpr (f == 2) store_k(Kw, kreg, kcodes, in4_k);
                    if constexpr (f == 3) {
                        if (in4_v) {
                            store_codes(Vw + st_v4, vcodes);
                        } else {
#pragma unroll
                            for (int i = 0; i < LD; ++i) *reinterpret_cast<u32x4_native*>(Vw + st_v + i * RPP * VROW) = vreg[i];
                        }
                        step_tile();
                    }
                    if constexpr (f == 4) load_tile(kreg, kcodes, kbase, k4, in4_k, pos_k, nv_k);
                    if constexpr (f == 5) load_tile(vreg, vcodes, vbase, v4, in4_v, pos_v, nv_v);
                }
                if constexpr (f == BAR) {
                    // K(j+2), V(j) are visible past this point: this wavefront's stores are done (seven
                    // or more later LDS accesses are behind them, LDS serves them in order), and every
                    // other one's too
                    __builtin_amdgcn_sched_barrier(0);
                    __builtin_amdgcn_s_waitcnt(0xC67F);      // lgkmcnt(6)
                    asm volatile("" ::: "memory");
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            psum = ps0 + ps1;
            __builtin_amdgcn_s_setprio(0);
            if constexpr (kind != kWhole4) {
                if (nv_next < BK) mask_tail(s, nv_next);
                nv_prev = nv_cur;
                nv_cur = nv_next;
                nv_next = nv_q1;          // of tile j + 2
            }
            ++j;
            raise = __any(psum > kTooBig);
        };
        // Inner loops = steady state.  They are left when a row sum shows that m must be raised; the outer
        // loop does that and re-enters.  (One loop for all kinds: 3425 against 3150 us for 12 x 128, 10200 rows on 40800 clean keys
        // and 20400 in slots.)
        for (;;) {
            bool finished = false;
            raise = false;
            if (j < whole4) {
                while (!raise && j < whole4) { lsum += psum; step(std::integral_constant<int, kWhole4>()); }
                // what step_tile() would have left: the last of these tiles may be the last of the range or of the clean region
                pos_q0 = t0 - BK; pos_q1 = t0 - 2 * BK;
                t0 -= BK;
                ++to_step;
                advance();
            }
            while (!raise && j < n4) { lsum += psum; step(std::integral_constant<int, kAny>()); }
            if (!raise) {
                do {
                    lsum += psum;
                    if (j == nt) { finished = true; break; }
                    step(std::integral_constant<int, kRows>());
                } while (!raise);
            }
            if (finished) break;
            // S of the tile just weighted again, its true row maximum, O and l to the new scale (the
            // products so far are in the old one), its weights anew
            f32x16_t y[2];
            qk(&sm.K[(j - 1) & 3][k_frag], y);
            if (nv_prev < BK) mask_tail(y, nv_prev);
            float v = fmaxf(y[0][0], y[1][0]);
#pragma unroll
            for (int i = 1; i < 16; ++i) v = fmaxf(v, fmaxf(y[0][i], y[1][i]));
            v = fmaxf(v, __shfl_xor(v, 32, FC_WAVE));
            const float mnew = fmaxf(m, v * c2);
            const float alpha = __builtin_amdgcn_exp2f(m - mnew);
            m = mnew;
            lsum *= alpha;
#pragma unroll
            for (int dv = 0; dv < DVB; ++dv) o[dv] *= alpha;
            ps0 = ps1 = 0.f;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const int kb = q >> 2, i = (q & 3) * 4;
                pack4(__builtin_amdgcn_exp2f(fmaf(y[kb][i], c2, -m)), __builtin_amdgcn_exp2f(fmaf(y[kb][i + 1], c2, -m)),
                      __builtin_amdgcn_exp2f(fmaf(y[kb][i + 2], c2, -m)), __builtin_amdgcn_exp2f(fmaf(y[kb][i + 3], c2, -m)), q);
            }
            psum = ps0 + ps1;
        }
        // ---- drain: O += V P of the last tile
        const bf16_t* Vl = &sm.V[(nt - 1) & 1][v_frag];
#pragma unroll
        for (int f = 0; f < NPV; ++f)
            o[f % DVB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f < PF ? frag[f] : read_v(Vl, f), __builtin_bit_cast(bf16x8_t, P[f / DVB]), o[f % DVB], 0, 0, 0);
    }

    // ---- epilogue: normalise, store O (bf16) and the row log-sum-exp; or leave the partial
    {
        const float ltot = lsum + __shfl_xor(lsum, 32, FC_WAVE);
        if (wi.S > 1) {
            const int64_t part = (wi.unit * (BQ / kUnitRows) + wave) * wi.S + wi.s;   // 32 rows each
            float* po = parts + (part * kUnitRows + l32) * D;
#pragma unroll
            for (int dv = 0; dv < DVB; ++dv)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    store_out(po + dv * 32 + g * 8 + hh * 4, o[dv][4 * g], o[dv][4 * g + 1], o[dv][4 * g + 2],
                              o[dv][4 * g + 3]);
            if (hh == 0) {
                float* ml = parts + (int64_t)p.parts * kUnitRows * D + part * 2 * kUnitRows;
                ml[l32] = m;
                ml[kUnitRows + l32] = ltot;
            }
            return;
        }
        const float inv = 1.0f / ltot;
        if (row_in_chunk < a.L_c) {
            const int64_t row = (int64_t)r * a.L_c + row_in_chunk;
            bf16_t* op = (bf16_t*)a.out + (row * a.H_q + h) * D;
#pragma unroll
            for (int dv = 0; dv < DVB; ++dv)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int e0 = dv * 32 + g * 8 + hh * 4;
                    store_out(op + e0, o[dv][4 * g] * inv, o[dv][4 * g + 1] * inv, o[dv][4 * g + 2] * inv,
                              o[dv][4 * g + 3] * inv);
                }
            if (a.lse && hh == 0)
                a.lse[(int64_t)h * a.A * a.L_c + row] =
                    (m + __builtin_amdgcn_logf(ltot)) * 0.6931471805599453f;
        }
    }
}

// ---- few query rows ---------------------------------------------------------------------
// 32 query rows per block; its 8 wavefronts take every 8th 32-key tile of the range and never meet before the end.  What bounds
// it are the bytes of the clean region and the latency of fetching them, so a wavefront has the codes of two tiles on their way
// while it works on a third, and K never passes through LDS: a lane holds half a row (hh: which half) of the key that the
// product's operand wants of it, if step st of the contraction is taken over elements hh D/2 + 8 st .. + 8 of both operands.
// V has to be transposed: bf16 rows in LDS, 16-byte pieces of a row exchanged (by the row's number) so that a lane can
// write its half row, and a transposing read fetch four rows' 32 bytes, without bank conflicts.
template <int D>
struct Narrow4Smem {
    static constexpr int OROW = D + 4;
    __attribute__((aligned(16))) union {
        struct { bf16_t v[kSplitWaves][32 * D], k[kSplitWaves][32 * D]; } t;   // one tile per wavefront; K of slots alone
        float o[kSplitWaves * kUnitRows * OROW];        // partial O at the end
    };
    float m_s[kSplitWaves * kUnitRows], l_s[kSplitWaves * kUnitRows];
    Segments sg;
};

template <int D>
__device__ __forceinline__ void attend_narrow4(const FcAttendArgs& a, const FcAttendPlan& p, uint32_t valid,
                                               Narrow4Smem<D>& sm, float* parts, const FcKv4& x) {
    constexpr int KS = D / 16;           // contraction steps of Q K^T
    constexpr int DVB = D / 32;          // 32-wide blocks of the value dimension
    constexpr int OROW = Narrow4Smem<D>::OROW;
    constexpr int VPR = D / 8;           // 16-byte vectors per row
    constexpr int LD = 32 * VPR / FC_WAVE;
    constexpr float kSlack = 8.0f;       // the exponents' reference follows the row maximum at this distance (log2)
    Segments& sg = sm.sg;
    float *m_s = sm.m_s, *l_s = sm.l_s;

    const SplitItem it = split_item(a, p, valid, blockIdx.x);
    if (!it.ok) return;
    const int hk = it.h / (a.H_q / a.H_k);
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int l32 = lane & 31, hh = lane >> 5;
    const float c2 = a.scale * 1.4426950408889634f;
    if (tid == 0) list_segments(a, it.c, sg);

    // B operand of S^T = K Q^T: lane holds Q[q = l32][hh D / 2 + 8 step .. + 8)
    bf16x8_t qf[KS];
    {
        int rc = it.tile * kUnitRows + l32;
        if (rc > a.L_c - 1) rc = a.L_c - 1;
        const bf16_t* qp = (const bf16_t*)a.q + (((int64_t)it.r * a.L_c + rc) * a.H_q + it.h) * D + hh * (D / 2);
#pragma unroll
        for (int st = 0; st < KS; ++st) qf[st] = *reinterpret_cast<const bf16x8_t*>(qp + 8 * st);
    }
    __syncthreads();
    const int tiles4 = (x.L_clean + 31) / 32;
    const int nt = tiles4 + __builtin_amdgcn_readfirstlane(sg.tile0[sg.n]);
    const int t_end = (int)((int64_t)nt * (it.s + 1) / it.S);
    const int t_end4 = t_end < tiles4 ? t_end : tiles4;
    int t = (int)((int64_t)nt * it.s / it.S) + wave;

    f32x16_t o[DVB];
#pragma unroll
    for (int b = 0; b < DVB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
    float m = kNegBig, l = 0.f;

    bf16_t *kw = sm.t.k[wave], *vw = sm.t.v[wave];
    // transposing reads of V: the lane's key row of the first 4-key patch, and its piece there; what depends on the patch and
    // on the block of the value dimension is exchanged into it
    const int l16 = lane & 15, v_row = hh * 4 + (l16 >> 2);
    const int v_at = v_row * D + fc_swapped<D>(v_row, ((lane >> 4) & 1) * 2 + ((l16 & 3) >> 1)) * 8 + (l16 & 1) * 4;

    // scores of one tile in s, V in LDS: weights, O, l
    auto weigh = [&](f32x16_t& s, int nv) {
        if (nv < 32) {
            const int mine = nv - hh * 4;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if ((i >> 2) * 8 + (i & 3) >= mine) s[i] = kNegBig;
        }
        float mx = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
        mx = fmaxf(mx, __shfl_xor(mx, 32, FC_WAVE)) * c2;
        if (__any(mx > m + kSlack)) {
            const float mn = fmaxf(m, mx);
            const float alpha = __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= alpha;
#pragma unroll
            for (int b = 0; b < DVB; ++b) o[b] *= alpha;
        }
        const float mneg = -m;
        const bf16x2_t ones = {(__bf16)1.0f, (__bf16)1.0f};
        bf16x8_t pf[2];
        float l0 = 0.f, l1 = 0.f;
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(s[i], c2, mneg));
            const float p1 = __builtin_amdgcn_exp2f(fmaf(s[i + 1], c2, mneg));
            const float p2 = __builtin_amdgcn_exp2f(fmaf(s[i + 2], c2, mneg));
            const float p3 = __builtin_amdgcn_exp2f(fmaf(s[i + 3], c2, mneg));
            const bf16x2_t lo = {(__bf16)p0, (__bf16)p1}, hi = {(__bf16)p2, (__bf16)p3};
            // the sums run over the rounded weights, the ones V is multiplied with
            l0 = __builtin_amdgcn_fdot2_f32_bf16(lo, ones, l0, false);
            l1 = __builtin_amdgcn_fdot2_f32_bf16(hi, ones, l1, false);
            pf[i >> 3][i & 7] = lo[0];
            pf[i >> 3][(i & 7) + 1] = lo[1];
            pf[i >> 3][(i & 7) + 2] = hi[0];
            pf[i >> 3][(i & 7) + 3] = hi[1];
        }
        l += l0 + l1;
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int b = 0; b < DVB; ++b) {
                // (rows + 8: the other half of the exchange's bits; blocks: pieces + 4 b)
                const s16x4_t lo = lds_read_tr(vw + ((v_at ^ (b * 32)) + tt * 16 * D));
                const s16x4_t hi = lds_read_tr(vw + ((v_at ^ (b * 32) ^ 8) + (tt * 16 + 8) * D));
                const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[tt], o[b], 0, 0, 0);
            }
    };

    // ---- tiles of codes
    const FcCodesHead head{x.k + (int64_t)hk * x.head_codes, x.v + (int64_t)hk * x.head_codes,
                           x.scales_at + (int64_t)hk * (x.head_scales - x.head_codes), x.L_clean, tiles4};
    const int st_row = l32 * D, st_swap = fc_swapped<D>(l32, hh * (D / 16)) * 8;
    auto codes_tile = [&](FcCodes<D>& c, int tt) {
        f32x16_t s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int st = 0; st < KS; ++st)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, c.key(st)), qf[st], s, 0, 0, 0);
        // the wavefront's own tile: its LDS accesses are served in order, no barrier is needed
#pragma unroll
        for (int st = 0; st < KS; ++st) *reinterpret_cast<u32x4_native*>(&vw[st_row + (st_swap ^ (st * 8))]) = c.value(st);
        const int nv = x.L_clean - tt * 32 < 32 ? x.L_clean - tt * 32 : 32;
        c.fetch(head, tt + 2 * kSplitWaves, l32, hh);
        weigh(s, nv);
    };
    if (t < t_end4) {
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

    // ---- tiles of the slots' rows
    u32x4_native kr[LD], vr[LD];
    int seg = 0, nvalid = 0;
    const bf16_t* kbase = (const bf16_t*)a.k_cache + (int64_t)hk * a.head_stride;
    const bf16_t* vbase = (const bf16_t*)a.v_cache + (int64_t)hk * a.head_stride;
    const uint32_t ts = (uint32_t)a.tok_stride;
    const int ld_row = lane / VPR, ld_col = lane % VPR;
    // tile tt -> registers, by rows; a row past the end of its segment re-reads the last one
    auto fetch = [&](int tt) {
        tt -= tiles4;
        while (tt >= __builtin_amdgcn_readfirstlane(sg.tile0[seg + 1])) ++seg;
        const int off = (tt - __builtin_amdgcn_readfirstlane(sg.tile0[seg])) * 32;
        const int left = __builtin_amdgcn_readfirstlane(sg.len[seg]) - off;
        const int64_t pos = (int64_t)(__builtin_amdgcn_readfirstlane(sg.start[seg]) + off) * a.tok_stride;
        nvalid = left < 32 ? left : 32;
        const char* kt = reinterpret_cast<const char*>(kbase + pos);
        const char* vt = reinterpret_cast<const char*>(vbase + pos);
#pragma unroll
        for (int i = 0; i < LD; ++i) {
            int row = i * (FC_WAVE / VPR) + ld_row;
            row = row < nvalid ? row : nvalid - 1;
            const uint32_t at = ((uint32_t)row * ts + 8u * (uint32_t)ld_col) * 2u;
            kr[i] = *reinterpret_cast<const u32x4_native*>(kt + at);
            vr[i] = *reinterpret_cast<const u32x4_native*>(vt + at);
        }
    };
    if (t < t_end) fetch(t);
    while (t < t_end) {
#pragma unroll
        for (int i = 0; i < LD; ++i) {
            const int row = i * (FC_WAVE / VPR) + ld_row, at = row * D + fc_swapped<D>(row, ld_col) * 8;
            *reinterpret_cast<u32x4_native*>(&kw[at]) = kr[i];
            *reinterpret_cast<u32x4_native*>(&vw[at]) = vr[i];
        }
        const int nv = nvalid;
        t += kSplitWaves;
        if (t < t_end) fetch(t);                        // the next tile, behind all of this one
        f32x16_t s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int st = 0; st < KS; ++st) {
            const bf16x8_t kf = *reinterpret_cast<const bf16x8_t*>(&kw[st_row + (st_swap ^ (st * 8))]);
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[st], s, 0, 0, 0);
        }
        weigh(s, nv);
    }

    l += __shfl_xor(l, 32, FC_WAVE);
    __syncthreads();                                    // every wavefront is done with its V tile
    if (hh == 0) { m_s[wave * kUnitRows + l32] = m; l_s[wave * kUnitRows + l32] = l; }
#pragma unroll
    for (int b = 0; b < DVB; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4_t*>(&sm.o[(wave * kUnitRows + l32) * OROW + b * 32 + g * 8 + hh * 4]) =
                f32x4_t{o[b][4 * g], o[b][4 * g + 1], o[b][4 * g + 2], o[b][4 * g + 3]};
    __syncthreads();
    finish_unit<bf16_t, D, OROW>(a, p, it, sm.o, m_s, l_s, parts);
}

// WIDE and NARROW say which of the two bodies some recompute count of this launch asks for.
template <int D, bool WIDE, bool NARROW>
__global__ __launch_bounds__(NT) void attend_kv4_kernel(FcAttendArgs a, FcAttendPlan p, float* parts, FcKv4 x) {
    static_assert(NT == kSplitThreads, "both bodies run on the same block");
    const uint32_t valid = valid_blocks(a);
    const int R = __popc(valid);
    if (R == 0) return;
    union Smem {
        WideSmem<WIDE ? D : 64> w;
        Narrow4Smem<NARROW ? D : 64> n;
    };
    __shared__ __attribute__((aligned(16))) char raw[WIDE && NARROW ? sizeof(Smem) : WIDE ? sizeof(WideSmem<D>) : sizeof(Narrow4Smem<D>)];
    if (WIDE && (!NARROW || !p.narrow[R - 1]))
        attend_wide4<D>(a, p, valid, *reinterpret_cast<WideSmem<D>*>(raw), parts, x);
    else if (NARROW)
        attend_narrow4<D>(a, p, valid, *reinterpret_cast<Narrow4Smem<D>*>(raw), parts, x);
}

template <int D>
int launch_kv4(FcAttendArgs a, const FcKv4& x, hipStream_t s) {
    a.L_clean = 0;                    // the slots alone
    FcAttendPlan p = fc_attend_plan_kv4(a.A, a.L_c, x.L_clean, a.H_q, D, true);
    if (!fc_room_for_partials(a.ws, a.ws_bytes, p.parts, D)) p = fc_attend_plan_kv4(a.A, a.L_c, x.L_clean, a.H_q, D, false);
    bool wide = false, narrow = false;
    for (int R = 0; R < a.A; ++R) (p.narrow[R] ? narrow : wide) = true;
    if (!narrow)
        attend_kv4_kernel<D, true, false><<<p.grid, NT, 0, s>>>(a, p, (float*)a.ws, x);
    else if (!wide)
        attend_kv4_kernel<D, false, true><<<p.grid, NT, 0, s>>>(a, p, (float*)a.ws, x);
    else
        attend_kv4_kernel<D, true, true><<<p.grid, NT, 0, s>>>(a, p, (float*)a.ws, x);
    FC_LAUNCH_CHECK();
    return launch_merge4<bf16_t, D>(a, p, s);
}

}  // namespace

int fc_launch_attend_kv4(const FcAttendArgs& a, const FcKv4& x, hipStream_t s) {
    if (a.d == 128) return launch_kv4<128>(a, x, s);
    if (a.d == 64) return launch_kv4<64>(a, x, s);
    return FC_UNSUPPORTED;
}
