// The MXFP4 product for few tiles (included by linear.hip, inside its namespace).
#pragma once

// 128 x 128 tiles, 8 waves of 64 x 32, one tile a workgroup.  Where a CU has a tile or two in all, nothing hides the way from memory but the
// transfers' own depth: a ring of three units of 256 contraction elements in LDS, two of which are on their way while one is multiplied (with the next
// stage in registers, one ahead, a unit takes 1.2 to 1.6 us where the weights come from memory; here 0.7, from memory 1.1).
// What bounds it: LDS, 0.43 us a unit, and meeting once a unit; from memory the weights' rows, of which a unit takes 128 bytes each.  Tried: a ring of four,
// 512 rows of 4096 x 4096 20.9 us for 20.4; the weights from memory straight into registers, four units ahead, and the rows through registers into
// LDS, 4 waves of 128 x 32: 24.9.
// LDS: a unit is A's and B's codes as in the streamed units (mx_tile.h), 128 rows each, then the scales of both, a row's eight bytes as they are.  LOOSE:
// scale rows that are not whole words come as the four words around them, and are shifted into place where they are read.  (A word that holds a byte of the
// row may be read whole: no word without one is.)
#define MXD_RING 3
#define MXD_CODES 16384
constexpr int mxd_unit(bool loose) { return 2 * MXD_CODES + (loose ? 4096 : 2048); }
constexpr int mxd_lds(bool loose) { return MXD_RING * mxd_unit(loose); }

// BLOCKS: K is not a multiple of the unit; what its last one lacks are other blocks of the row, and zeros where A's fragments are used
template <bool LOOSE, bool BLOCKS, typename END>
__global__ void __launch_bounds__(512, 2)
k_mxfp4_deep(MxOperand A, MxOperand B, int nblk, MxOrder order, END end) {
    constexpr bool PARTS = std::is_same<END, MxParts>::value;
    constexpr int UNIT = mxd_unit(LOOSE), DMA = LOOSE ? 6 : 5;           // transfers a wave makes for a unit
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wa = wave >> 2, wb = wave & 3;
    const int lane = (int)threadIdx.x & 63, li = lane & 31, half = lane >> 5;
    int tm, tn;
    if (order.bands.group > 0) tile_coords(order.bands, tm, tn);
    else tile_coords(order.regions, tm, tn);
    const int64_t m0 = 128 * (int64_t)tm, n0 = 128 * (int64_t)tn;
    int first = 0, niter = (nblk + 7) / 8;
    if constexpr (PARTS) {
        first = end.units * (int)blockIdx.y;
        niter = niter - first < end.units ? niter - first : end.units;
    }
    const uint32_t cstride = 16u * (uint32_t)nblk, sstride = (uint32_t)nblk;

    // ---- transfers: the lane's rows and segments; rows past the operand's end are its last row once more
    const int ta = (int)(A.rows - m0 < 128 ? A.rows - m0 : 128) - 1, tb = (int)(B.rows - n0 < 128 ? B.rows - n0 : 128) - 1;
    uint32_t ra[2], rb[2];
    int sg[2];
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        const int row = 16 * wave + 8 * v + (lane >> 3);
        ra[v] = (uint32_t)(row < ta ? row : ta) * cstride;
        rb[v] = (uint32_t)(row < tb ? row : tb) * cstride;
        sg[v] = (lane & 7) ^ (lane >> 4) ^ (4 * v);
    }
    // scales: waves 0 .. 3 have A's rows, 4 .. 7 B's
    const uint8_t* const sbase = wave < 4 ? A.scales + m0 * sstride : B.scales + n0 * sstride;
    const int ts = wave < 4 ? ta : tb;
    const uint32_t off = (uint32_t)(uintptr_t)sbase & 3u;                           // of the scales from a word's start (LOOSE)
    uint32_t rs[LOOSE ? 2 : 1];
#pragma unroll
    for (int v = 0; v < (LOOSE ? 2 : 1); ++v) {
        const int row = 32 * (wave & 3) + (LOOSE ? 16 * v + (lane >> 2) : lane >> 1);
        rs[v] = (uint32_t)(row < ts ? row : ts) * sstride + (LOOSE ? off : 0u);
    }
    const uint8_t *pa = A.codes + m0 * cstride, *pb = B.codes + n0 * cstride;
    auto issue = [&](int it) GS_INLINE {
        const int u = first + it;
        const uint32_t buf = lds0 + (uint32_t)(it % MXD_RING) * UNIT;
        const uint8_t *qa = gs_uniform(pa + 128 * (int64_t)u), *qb = gs_uniform(pb + 128 * (int64_t)u), *qs = gs_uniform(sbase + 8 * (int64_t)u - (LOOSE ? off : 0u));
        const int have = BLOCKS ? nblk - 8 * u : 8;                                  // blocks of the unit
        uint32_t oa[2], ob[2];
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            const uint32_t seg = 16u * (uint32_t)(!BLOCKS || sg[v] < have ? sg[v] : 0);
            oa[v] = ra[v] + seg;
            ob[v] = rb[v] + seg;
        }
        const uint32_t dc = buf + 2048u * wave;
        gs_dma16<0>(dc, oa[0], qa);
        gs_dma16<1024>(dc, oa[1], qa);
        gs_dma16<MXD_CODES>(dc, ob[0], qb);
        gs_dma16<MXD_CODES + 1024>(dc, ob[1], qb);
        if constexpr (LOOSE) {
            // the word that holds the row's first byte and those behind it, as far as they hold any of the unit's; else the first once more
            const uint32_t ds = buf + 512u * wave;
            const uint32_t w0 = rs[0] & ~3u, w1 = rs[1] & ~3u, j = 4u * (lane & 3);
            gs_dma4<2 * MXD_CODES>(ds, j < (rs[0] & 3u) + (have < 8 ? have : 8) ? w0 + j : w0, qs);
            gs_dma4<2 * MXD_CODES + 256>(ds, j < (rs[1] & 3u) + (have < 8 ? have : 8) ? w1 + j : w1, qs);
        } else {
            const uint32_t b = 4u * (lane & 1);
            gs_dma4<2 * MXD_CODES>(buf + 256u * wave, rs[0] + (!BLOCKS || (int)b < have ? b : 0u), qs);
        }
    };

    float16_t acc[2][1];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][0][v] = 0.0f;
#pragma unroll
    for (int it = 0; it < MXD_RING - 1; ++it)
        if (it < niter) issue(it);
    uint32_t sh[3];                                      // how far a fragment's rows' scales are from a word's start (LOOSE)
#pragma unroll
    for (int x = 0; x < 3; ++x) {
        const int row = x < 2 ? 64 * wa + 32 * x + li : 32 * wb + li, most = x < 2 ? ta : tb;
        sh[x] = ((uint32_t)(uintptr_t)((x < 2 ? A.scales + m0 * sstride : B.scales + n0 * sstride)) + (uint32_t)(row < most ? row : most) * sstride) & 3u;
    }
    uint32_t ad[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) ad[s] = 128u * li + 16u * (uint32_t)((2 * s + half) ^ (li >> 1 & 7));
    auto unit = [&](int it, auto last_) GS_INLINE {
        constexpr bool last = decltype(last_)::value;
        const uint8_t* buf = lds + (it % MXD_RING) * UNIT;
        uvec4_t f[3][4];                                 // fragments of the four steps: 0 and 1 of A's rows, 2 of B's
        uint32_t sc[3][2];
#pragma unroll
        for (int x = 0; x < 3; ++x) {
            const int row = x < 2 ? 64 * wa + 32 * x : 32 * wb;
#pragma unroll
            for (int s = 0; s < 4; ++s) f[x][s] = *reinterpret_cast<const uvec4_t*>(buf + (x < 2 ? 0 : MXD_CODES) + 128 * row + ad[s]);
            const int srow = (x < 2 ? 0 : 128) + row + li;
            uvec2_t w;
            if constexpr (LOOSE) {
                const uvec4_t q = *reinterpret_cast<const uvec4_t*>(buf + 2 * MXD_CODES + 16 * srow);
                w.x = __builtin_amdgcn_alignbyte(q.y, q.x, sh[x]);
                w.y = __builtin_amdgcn_alignbyte(q.z, q.y, sh[x]);
            } else {
                w = *reinterpret_cast<const uvec2_t*>(buf + 2 * MXD_CODES + 8 * srow);
            }
            sc[x][0] = w.x >> (8 * half);                // bytes 0 and 2 are this lane's blocks
            sc[x][1] = w.y >> (8 * half);
        }
        if constexpr (last) {
            const int have = nblk - 8 * (first + it);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                if (2 * s + half < have) continue;
                f[0][s] = f[1][s] = uvec4_t{0u, 0u, 0u, 0u};
                if constexpr (LOOSE) {                   // (others' bytes: zeros under a scale that is no number would be none)
#pragma unroll
                    for (int x = 0; x < 3; ++x) sc[x][s >> 1] = (sc[x][s >> 1] & ~(0xFFu << (16 * (s & 1)))) | 0x7Fu << (16 * (s & 1));
                }
            }
        }
        gs_for<4>([&](auto sc_) GS_INLINE {
            constexpr int s = decltype(sc_)::value, sel = 2 * (s & 1);
            const int8v_t b = {(int)f[2][s].x, (int)f[2][s].y, (int)f[2][s].z, (int)f[2][s].w, 0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int8v_t a = {(int)f[i][s].x, (int)f[i][s].y, (int)f[i][s].z, (int)f[i][s].w, 0, 0, 0, 0};
                acc[i][0] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, a, acc[i][0], 4, 4, sel, (int)sc[2][s >> 1], sel, (int)sc[i][s >> 1]);
            }
        });
    };
    // a unit: its transfers have arrived and the ring's oldest buffer has been read by all, which then takes the transfers of the unit two on
    int it = 0;
#pragma unroll 1
    for (; it + MXD_RING - 1 < niter; ++it) {
        gs_meet<(MXD_RING - 2) * DMA>();
        issue(it + MXD_RING - 1);
        unit(it, std::false_type{});
    }
#pragma unroll 1
    for (; it < niter; ++it) {
        const int left = niter - 1 - it;
        if (left == 1) gs_meet<DMA>();
        else gs_meet<0>();
        if (BLOCKS && left == 0) unit(it, std::true_type{});
        else unit(it, std::false_type{});
    }
    gs_meet<0>();                                        // every wave has its fragments: the ring takes the rows on their way out
    static_assert(8 * mx_wave_rows<float, 1>() <= mxd_lds(LOOSE), "the staged rows fit the ring");
    if constexpr (PARTS)
        mx_store_wave<float, true, 2, 1>(acc, lds + wave * mx_wave_rows<float, 1>(), end.sums + end.stride * blockIdx.y, end.ld, m0 + 64 * wa,
                                         n0 + 32 * wb, A.rows, B.rows, true, m0 + 128 <= A.rows && n0 + 128 <= B.rows, lane);
    else
        mx_finish_wave<2, 1>(acc, lds + wave * mx_wave_rows<float, 1>(), end, m0 + 64 * wa, n0 + 32 * wb, A.rows, B.rows, lane);
}
