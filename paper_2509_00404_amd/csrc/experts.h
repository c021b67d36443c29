// The experts' slots on the device, and MXFP4 blocks: what the kernels of the experts' products share.
#pragma once
#include "elementwise.h"

#define EXPERTS_MAX 512
#define SLOT_ALIGN 256                    // segments of a matrix quantized along the slots have rows of whole units of this many

namespace {

// Where unit u lies when every expert's slots are cut into units of `size` (the last of an expert may be short, an expert without slots has
// none): the expert, its slots, and the unit's number among its own.  expert = -1 behind the last unit; `total` = units in all.  Every
// wave looks for itself, its lanes holding up to eight neighbouring experts.  Offsets are held to 0 <= o <= S and to ascend, whatever the
// memory says: one that is smaller than one before it counts as the largest before it, so that segments never overlap and all of them
// together are at most S slots.  (Whether any descends is one ballot; the scan that mends it runs only then.)
struct SlotUnit {
    int expert, local, total;
    int64_t begin, end;                   // the expert's slots
    int64_t used;                         // the end of all experts' slots
};
__device__ __forceinline__ int64_t held(int32_t o, int64_t S) { return o < 0 ? 0 : o > S ? S : o; }
__device__ __forceinline__ SlotUnit find_unit(const int32_t* __restrict__ offsets, int E, int64_t S, int size, int64_t u) {
    constexpr int Q = EXPERTS_MAX / 64;
    const int lane = (int)threadIdx.x & 63, q = (E + 63) >> 6, e0 = lane * q;
    int32_t o[Q + 1];
#pragma unroll
    for (int i = 0; i <= Q; ++i) {
        const int e = e0 + (i < q ? i : q);
        o[i] = offsets[e < E ? e : E];
    }
    int mine = 0;
    bool descends = false;
#pragma unroll
    for (int i = 0; i <= Q; ++i) {
        o[i] = (int32_t)held(o[i], S);
        descends |= i > 0 && o[i] < o[i > 0 ? i - 1 : 0];
    }
    if (__any(descends)) {
#pragma unroll
        for (int i = 1; i <= Q; ++i) o[i] = o[i] > o[i - 1] ? o[i] : o[i - 1];
        int32_t top = o[Q];
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int32_t a = __shfl_up(top, d);
            if (lane >= d && a > top) top = a;
        }
        const int32_t before = __shfl_up(top, 1);
#pragma unroll
        for (int i = 0; i <= Q; ++i) o[i] = lane > 0 && before > o[i] ? before : o[i];
    }
#pragma unroll
    for (int i = 0; i < Q; ++i) {
        const int32_t n = o[i + 1] - o[i];
        if (n > 0) mine += (n + size - 1) / size;
    }
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int a = __shfl_up(upto, d);
        if (lane >= d) upto += a;
    }
    SlotUnit r;
    r.total = __builtin_amdgcn_readlane(upto, 63);
    r.expert = -1;
    r.local = 0;
    r.begin = r.end = 0;
    r.used = __builtin_amdgcn_readlane(o[Q], 63);
    if (u >= r.total) return r;
    // every lane looks through its own experts, and the one that has the unit says where
    int before = upto - mine, expert = 0, local = 0, begin = 0, end = 0;
#pragma unroll
    for (int i = 0; i < Q; ++i) {
        const int32_t n = o[i + 1] - o[i], units = n > 0 ? (n + size - 1) / size : 0;
        const bool here = u >= before && u < before + units;
        expert = here ? e0 + i : expert;
        local = here ? (int)(u - before) : local;
        begin = here ? o[i] : begin;
        end = here ? o[i + 1] : end;
        before += units;
    }
    const int at = __ffsll((unsigned long long)__ballot(upto > u)) - 1;
    r.expert = __builtin_amdgcn_readlane(expert, at);
    r.local = __builtin_amdgcn_readlane(local, at);
    r.begin = __builtin_amdgcn_readlane(begin, at);
    r.end = __builtin_amdgcn_readlane(end, at);
    return r;
}
// expert e's slots, and the units of `size` of the experts before it (offsets held as above)
struct ExpertSlots {
    int64_t units_before, count;
};
__device__ __forceinline__ ExpertSlots slots_of(const int32_t* __restrict__ offsets, int E, int64_t S, int size, int e) {
    constexpr int Q = EXPERTS_MAX / 64;
    const int lane = (int)threadIdx.x & 63;
    int32_t o[Q][2];
#pragma unroll
    for (int i = 0; i < Q; ++i) {
        const int x = 64 * i + lane;                     // (those from e on: nothing)
        o[i][0] = offsets[x < e ? x : e];
        o[i][1] = offsets[x < e ? x + 1 : e];
    }
    int64_t begin = held(offsets[e], S), end = held(offsets[e + 1], S);
    bool descends = end < begin;
    int sum = 0;
#pragma unroll
    for (int i = 0; i < Q; ++i) {
        const int64_t n = held(o[i][1], S) - held(o[i][0], S);
        descends |= n < 0;
        if (n > 0) sum += (int)((n + size - 1) / size);
    }
    if (__any(descends)) {
        int64_t all = 0;
        begin = held(offsets[0], S);
        for (int x = 0; x < e; ++x) {
            end = held(offsets[x + 1], S);
            end = end > begin ? end : begin;
            all += (end - begin + size - 1) / size;
            begin = end;
        }
        end = held(offsets[e + 1], S);
        return {all, end > begin ? end - begin : 0};
    }
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) sum += __shfl_xor(sum, m);
    return {__builtin_amdgcn_readfirstlane(sum), end - begin};
}
// units of `size` that S slots can fall into
inline int64_t most_units(int64_t S, int E, int size) { return S / size + (E < S ? E : S); }

// MXFP4: X = 2^(floor(log2 amax) - 2) as its E8M0 byte, 1 / X, and eight codes: nearest, ties to the even one, saturated at 6
__device__ __forceinline__ uint32_t mx_scale(float amax) {
    const int field = (int)(__float_as_uint(amax) >> 23);
    return field > 2 ? (field < 255 ? field - 2 : 254) : 0;
}
__device__ __forceinline__ float mx_inverse(uint32_t byte) { return __uint_as_float(byte < 254u ? (254u - byte) << 23 : 0x400000u); }
__device__ __forceinline__ uint32_t mx_pack8(float a, float b, float c, float d, float e, float f, float g, float h) {
    uint32_t w = 0u;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a, b, 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, c, d, 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e, f, 1.0f, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, g, h, 1.0f, 3);
}
// eight elements of a block that four lanes hold: their codes, and the block's scale
__device__ __forceinline__ uint32_t mx_quad(const float (&v)[8], uint32_t& byte) {
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(v[i]));
    amax = fmaxf(amax, __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(amax), 0xB1, 0xF, 0xF, true)));    // lanes 1 0 3 2
    amax = fmaxf(amax, __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(amax), 0x4E, 0xF, 0xF, true)));    // lanes 2 3 0 1
    byte = mx_scale(amax);
    const float inv = mx_inverse(byte);
    return mx_pack8(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv, v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
}
// one block of a lane's own
__device__ __forceinline__ ew_u4 mx_block(const float (&v)[32], uint32_t& byte) {
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) amax = fmaxf(amax, fabsf(v[i]));
    byte = mx_scale(amax);
    const float inv = mx_inverse(byte);
    ew_u4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = mx_pack8(v[8 * i] * inv, v[8 * i + 1] * inv, v[8 * i + 2] * inv, v[8 * i + 3] * inv, v[8 * i + 4] * inv, v[8 * i + 5] * inv,
                        v[8 * i + 6] * inv, v[8 * i + 7] * inv);
    return w;
}

}  // namespace
