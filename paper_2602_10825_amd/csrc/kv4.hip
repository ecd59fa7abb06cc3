// Rows of the K/V cache to 4 bits and back (the format: kv4.hpp).
#include "kv4.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kPasses = 2;             // of a packing: rows of a lane that are read before the first is worked on
// An unpacking that writes more than this streams its output past the caches (the Infinity Cache holds 256 MB).  bf16 rows,
// unpacked / unpacked and their importance taken, streamed against not: 250 MB 50.5 : 67.9 / 102 : 115 us, 920 MB 168 : 226 / 391 : 426,
// 184 MB 38.7 : 39.8 / 81.7 : 80.1, 61 MB 16.8 : 18.7 / 46.4 : 44.4.
constexpr int64_t kStreamFrom = 200ll << 20;

// The largest value over the four lanes of a block (lanes 4 i .. 4 i + 3).
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);        // quad_perm 1 0 3 2
    v = v > o ? v : o;
    o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);                 // quad_perm 2 3 0 1
    return v > o ? v : o;
}

// A lane has the EPL elements of one row that are 16 bytes of the cache.
template <typename T>
struct Lane {
    static constexpr int EPL = Elem<T>::kVec, LPB = 32 / EPL;       // lanes per block of 32: 4 (bf16) or 8 (fp32)
};
template <int LPB>
__device__ __forceinline__ uint32_t block_max(uint32_t v) {
    v = quad_max(v);
    if (LPB == 8) {
        const uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true);     // the other quad of eight
        v = v > o ? v : o;
    }
    return v;
}

// The scale's exponent: of the block's largest magnitude, as a float's bits, the exponent less 2; less 1 from 1.75 times its power
// of two on, which adding a quarter to the fraction carries over.  Then the largest code is 4 or 6, except that magnitudes of
// 1.75 2^127 and more, whose scale would make 4 an infinity, take 6 (and so does everything above 1.5 2^127).  On N(0, 1) this border
// leaves an error of 0.1118 of a standard deviation, 2 (no exception) 0.1149, 1.5 (nothing is ever cut off) 0.1154.  Packing what a
// packed block stands for gives the same block.
// Bound by HBM: 24 x 128, K and V of 37440 kept rows of 74880 (460 MB read, 122 written) 107 us, 5.4 TB/s.  Read
// past the caches (the call 245 -> 226 us with the unpacking behind it: what is read next are the packed rows); two rows a lane
// instead of one 258 -> 245, four or eight no more.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void kv4_pack_kernel(FcKv4Args a) {
    constexpr int EPL = Lane<T>::EPL, LPB = Lane<T>::LPB, LPR = D / EPL, RPW = FC_WAVE / LPR;      // lanes per row, rows per wavefront and pass
    const int h = blockIdx.y;
    const T* src = (const T*)(blockIdx.z ? a.v_cache : a.k_cache) + h * a.head_stride;
    uint8_t* codes = (blockIdx.z ? a.v4 : a.k4) + (int64_t)h * a.capacity4 * (D / 2);
    uint8_t* scales = (blockIdx.z ? a.v4 : a.k4) + a.H_k * a.capacity4 * (D / 2) + (int64_t)h * a.capacity4 * (D / 32);
    const int lane = threadIdx.x & 63, l = lane % LPR;
    const int i0 = ((blockIdx.x * (kThreads / FC_WAVE) + (threadIdx.x >> 6)) * kPasses) * RPW + lane / LPR;
    float f[kPasses][EPL];
    bool ok[kPasses];
#pragma unroll
    for (int e = 0; e < kPasses; ++e) {
        const int i = i0 + e * RPW;
        ok[e] = i < a.count;
        int64_t row = a.cache_pos + (int64_t)(ok[e] ? i : 0);
        if (a.kept) {
            row = a.kept[(int64_t)h * a.count + (ok[e] ? i : 0)];
            const bool inside = (uint64_t)row < (uint64_t)a.L_k;     // else skipped: the 4-bit row stays as it was
            ok[e] = ok[e] && inside;
            row = inside ? row : 0;
        }
        unpack16(nt_load16(reinterpret_cast<const uint4*>(src + row * a.tok_stride + EPL * l)), f[e], T());
    }
#pragma unroll
    for (int e = 0; e < kPasses; ++e) {
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < EPL; ++k) {
            const uint32_t u = __float_as_uint(f[e][k]) & 0x7fffffffu;
            top = u > top ? u : top;
        }
        top = block_max<LPB>(top);
        const bool finite = top < 0x7f800000u;
        int byte = (int)((top + 0x200000u) >> 23) - 2;
        byte = byte < 1 ? 1 : (byte > 252 ? 252 : byte);
        const float s = __uint_as_float((uint32_t)byte << 23);
        byte = finite ? byte : 255;
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[e][0], f[e][1], s, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[e][2], f[e][3], s, 1);
        if constexpr (EPL == 8) {
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[e][4], f[e][5], s, 2);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[e][6], f[e][7], s, 3);
        }
        w = finite ? w : 0u;
        if (!ok[e]) continue;
        const int64_t to = a.pos4 + (int64_t)(i0 + e * RPW);
        if constexpr (EPL == 8) *reinterpret_cast<uint32_t*>(codes + to * (D / 2) + 4 * l) = w;
        else *reinterpret_cast<uint16_t*>(codes + to * (D / 2) + 2 * l) = (uint16_t)w;
        if (l % LPB == 0) scales[to * (D / 32) + l / LPB] = (uint8_t)byte;
    }
}

// EPL codes and their scale's byte -> 16 bytes of the cache
__device__ __forceinline__ u32x4_native expand(uint32_t codes, uint32_t scale, bf16_t) { return fc_kv4_to_bf16(codes, scale); }
__device__ __forceinline__ u32x4_native expand(uint32_t codes, uint32_t scale, float) { return __builtin_bit_cast(u32x4_native, fc_kv4_to_f32(codes, scale)); }

template <typename T, int D, bool STREAM>
__global__ __launch_bounds__(kThreads) void kv4_unpack_kernel(FcKv4Args a) {
    constexpr int EPL = Lane<T>::EPL, LPB = Lane<T>::LPB, LPR = D / EPL;
    const int h = blockIdx.y;
    T* dst = (T*)(blockIdx.z ? a.v_cache : a.k_cache) + h * a.head_stride;
    const uint8_t* codes = (blockIdx.z ? a.v4 : a.k4) + (int64_t)h * a.capacity4 * (D / 2);
    const uint8_t* scales = (blockIdx.z ? a.v4 : a.k4) + a.H_k * a.capacity4 * (D / 2) + (int64_t)h * a.capacity4 * (D / 32);
    const int i = blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR, l = threadIdx.x % LPR;
    if (i >= a.count) return;
    const int64_t from = a.pos4 + (int64_t)i;
    uint32_t w;
    if constexpr (EPL == 8) w = *reinterpret_cast<const uint32_t*>(codes + from * (D / 2) + 4 * l);
    else w = *reinterpret_cast<const uint16_t*>(codes + from * (D / 2) + 2 * l);
    const u32x4_native v = expand(w, scales[from * (D / 32) + l / LPB], T());
    u32x4_native* to = reinterpret_cast<u32x4_native*>(dst + (a.cache_pos + (int64_t)i) * a.tok_stride + EPL * l);
    if constexpr (STREAM) __builtin_nontemporal_store(v, to);
    else *to = v;
}

template <typename T, int D>
int launch(const FcKv4Args& a, bool pack, hipStream_t s) {
    const int64_t rows = kThreads / (D / Lane<T>::EPL) * (pack ? kPasses : 1);
    const dim3 grid((unsigned)((a.count + rows - 1) / rows), a.H_k, a.v_cache ? 2 : 1);
    const int64_t written = (int64_t)a.count * a.H_k * D * sizeof(T) * (a.v_cache ? 2 : 1);
    if (pack)
        kv4_pack_kernel<T, D><<<grid, kThreads, 0, s>>>(a);
    else if (written > kStreamFrom)
        kv4_unpack_kernel<T, D, true><<<grid, kThreads, 0, s>>>(a);
    else
        kv4_unpack_kernel<T, D, false><<<grid, kThreads, 0, s>>>(a);
    FC_LAUNCH_CHECK();
    return FC_OK;
}

int launch_any(const FcKv4Args& a, bool pack, hipStream_t s) {
    if (a.count == 0) return FC_OK;
    if (a.dtype == FC_BF16) return a.d == 128 ? launch<bf16_t, 128>(a, pack, s) : launch<bf16_t, 64>(a, pack, s);
    return a.d == 128 ? launch<float, 128>(a, pack, s) : launch<float, 64>(a, pack, s);
}

}  // namespace

int fc_launch_kv4_pack(const FcKv4Args& a, hipStream_t s) { return launch_any(a, true, s); }
int fc_launch_kv4_unpack(const FcKv4Args& a, hipStream_t s) { return launch_any(a, false, s); }
