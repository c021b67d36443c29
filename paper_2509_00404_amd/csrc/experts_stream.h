// The experts' products for many slots: one stream of units over ragged tiles (included by experts.hip, inside its namespace).
#pragma once

// The tiles and units are those of the dense MXFP4 stream: 256 x 256 outputs by 8 waves of 128 x 64, a unit of 256 contraction elements
// of both operands goes straight into one of two LDS buffers while the other is multiplied, and the next tile's units travel while this
// one ends.  What is different is where tiles lie and how long they are, which the device alone knows:
//   EX_PRODUCT  C[s, n]: the expert's slots against its N outputs; its last tile of slots is short.  The first operand's rows are the
//               slots', or the tokens' by way of token[]: those of the next tile are fetched while this one is multiplied.
//   EX_WGRAD    dW_e[n, k] over the expert's slots: every tile whole, the contraction as long as the expert has slots.
// A workgroup works its way through the tiles, gridDim.x apart.  Neighbouring tiles are of one expert, up to EX_BAND of its column tiles wide,
// and every XCD works on a run of them: they share panels of both operands in its L2.
// A wave whose 128 rows lie behind the tile's end multiplies nothing, and a last unit that exists in part is multiplied by steps of 64.
#define EX_BAND 8
enum { EX_PRODUCT = 0, EX_WGRAD = 1 };
struct ExStream {
    MxRows A, B;                          // first operand (slots, or N), second (weights, or K)
    const int32_t* offsets;
    const int32_t* token;                 // null: rows by slot
    int64_t S, arows;                     // slots; rows of A
    int64_t N;                            // product: outputs of an expert; gradient: N
    int64_t K;                            // product: contraction, a multiple of 32; gradient: K
    uint32_t astride;                     // product: bytes of a row of A's codes, a multiple of 128 (its tail is zeros)
    uint32_t bscales;                     // product: bytes of a row of B's scales, a multiple of 8
    int E, tiles_m, tiles_n;              // gradient: tiles_m along N, tiles_n along K; product: tiles_n along N
};
#define EX_LDS (MXS_LDS + 4 * 4 * (EXPERTS_MAX + 1))     // behind the two buffers what every expert has, four numbers

// zeros to n elements from p
template <typename OUT>
__device__ __forceinline__ void ex_clear(OUT* p, int64_t n, bool vec) {
    constexpr int E = 16 / (int)sizeof(OUT);
    const int64_t units = vec ? n / E : 0;
    for (int64_t c = threadIdx.x; c < units; c += 512) reinterpret_cast<uvec4_t*>(p)[c] = uvec4_t{0u, 0u, 0u, 0u};
    for (int64_t c = units * E + threadIdx.x; c < n; c += 512) p[c] = OUT(0);
}

template <typename OUT, int MODE>
__global__ void __launch_bounds__(512, 2)
k_experts_stream(ExStream a, OUT* __restrict__ C, int64_t ldc, bool vec) {
    constexpr bool LINES = sizeof(OUT) == 2;             // outputs by way of LDS, accumulator tiles transposed
    constexpr bool WGRAD = MODE == EX_WGRAD;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    int32_t* const s_first = reinterpret_cast<int32_t*>(lds + MXS_LDS);              // first tile of every expert, and their number
    int32_t* const s_begin = s_first + EXPERTS_MAX + 1;                              // an expert's first slot,
    int32_t* const s_count = s_begin + EXPERTS_MAX + 1;                              // its slots,
    int32_t* const s_padded = s_count + EXPERTS_MAX + 1;                             // and segments of SLOT_ALIGN before it
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wa = wave >> 2, wb = wave & 3;
    const int lane = (int)threadIdx.x & 63, li = lane & 31, half = lane >> 5;

    // ---- the tables, by every expert's thread
    {
        const int e = (int)threadIdx.x;
        int64_t n = 0;
        if (e < a.E) {
            const int64_t b = held(a.offsets[e], a.S);
            n = held(a.offsets[e + 1], a.S) - b;
            if (n < 0) n = 0;
            s_begin[e] = (int32_t)b;
            s_count[e] = (int32_t)n;
        }
        int tiles = WGRAD ? (n > 0 ? a.tiles_m * a.tiles_n : 0) : (int)((n + 255) >> 8) * a.tiles_n, segs = (int)((n + SLOT_ALIGN - 1) / SLOT_ALIGN);
        int32_t* s_sum = reinterpret_cast<int32_t*>(lds);                            // (the waves' sums, before any unit is here)
        const int mine_t = tiles, mine_s = segs;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int t = __shfl_up(tiles, d), g = __shfl_up(segs, d);
            if (lane >= d) { tiles += t; segs += g; }
        }
        if (lane == 63) { s_sum[wave] = tiles; s_sum[8 + wave] = segs; }
        __syncthreads();
        for (int w = 0; w < wave; ++w) { tiles += s_sum[w]; segs += s_sum[8 + w]; }
        if (e < a.E) { s_first[e] = tiles - mine_t; s_padded[e] = segs - mine_s; }
        if (e == a.E - 1) s_first[a.E] = tiles;
        __syncthreads();
    }
    const int total = __builtin_amdgcn_readfirstlane(s_first[a.E]);
    auto begin_of = [&](int e) GS_INLINE { return __builtin_amdgcn_readfirstlane(s_begin[e]); };
    auto count_of = [&](int e) GS_INLINE { return __builtin_amdgcn_readfirstlane(s_count[e]); };

    // ---- what no tile covers
    if constexpr (WGRAD) {
        for (int e = 0; e < a.E; ++e)                                                // experts without slots
            if (count_of(e) == 0)
                for (int64_t r = blockIdx.x; r < a.N; r += gridDim.x) ex_clear(C + ((int64_t)e * a.N + r) * ldc, a.K, vec);
    } else {
        for (int64_t r = (int64_t)begin_of(a.E - 1) + count_of(a.E - 1) + blockIdx.x; r < a.S; r += gridDim.x)      // slots that serve no choice
            ex_clear(C + r * ldc, a.N, vec);
    }

    // tile number -> expert (searched on from e) and place
    auto tile_of = [&](int tile, int& e, int& m0, int& n0) GS_INLINE {
        while (tile >= __builtin_amdgcn_readfirstlane(s_first[e + 1])) ++e;
        const int first = __builtin_amdgcn_readfirstlane(s_first[e]), local = tile - first;
        const int down = WGRAD ? a.tiles_m : (count_of(e) + 255) >> 8;
        const int band = local / (EX_BAND * down), r = local - band * EX_BAND * down;
        const int left = a.tiles_n - band * EX_BAND, w = left < EX_BAND ? left : EX_BAND;
        const int tm = r / w;
        m0 = 256 * tm;
        n0 = 256 * (band * EX_BAND + r - tm * w);
    };
    const int hop = (int)gridDim.x, xcds = (hop & 7) == 0 ? 8 : 1;
    const int start = ((int)blockIdx.x % xcds) * (hop / xcds) + (int)blockIdx.x / xcds;
    if (start >= total) return;

    // ---- transfers
    const uint8_t *qa, *qb, *qsa, *qsb;                  // the next unit's codes and scales
    int lpos = start, lcnt = 0, lblk = 8;                // tile being fetched, units left of it, blocks of 32 of the unit that B has
    uint32_t va[4], vb[4], wsa, wsb;                     // the lane's offsets
    int32_t row_next[5];                                 // rows of A of the tile to be entered next, by this lane's place
    int nexp = 0, nm0 = 0, nn0 = 0;                      // that tile
    auto look_ahead = [&](int pos) GS_INLINE {
        tile_of(pos < total ? pos : total - 1, nexp, nm0, nn0);
        if constexpr (!WGRAD) {
            const int l = gs_fresh_lane();
            const int32_t b = begin_of(nexp) + nm0, t = count_of(nexp) - nm0 - 1;
#pragma unroll
            for (int v = 0; v < 5; ++v) {
                const int row = v < 4 ? 32 * wave + 8 * v + (l >> 3) : 32 * wave + (l >> 1);
                row_next[v] = b + (row < t ? row : t);
                if (a.token) row_next[v] = a.token[row_next[v]];
            }
        }
    };
    auto enter = [&]() GS_INLINE {
        const int e = nexp, m0 = nm0, n0 = nn0;
        const int l = gs_fresh_lane();
        const uint32_t seg0 = (uint32_t)((l & 7) ^ (l >> 4)) * 16;
        const int64_t brows = WGRAD ? a.K : a.N;
        const int tb = (int)(brows - n0 < 256 ? brows - n0 : 256) - 1;
        const int rs = 32 * wave + (l >> 1);
        if constexpr (WGRAD) {
            const int len = (count_of(e) + SLOT_ALIGN - 1) / SLOT_ALIGN * SLOT_ALIGN;
            const int64_t at = (int64_t)__builtin_amdgcn_readfirstlane(s_padded[e]) * SLOT_ALIGN;
            const int64_t pa = at * a.N + (int64_t)m0 * len, pb = at * a.K + (int64_t)n0 * len;
            lcnt = (count_of(e) + 255) >> 8;
            qa = a.A.codes + pa / 2;
            qsa = a.A.scales + pa / 32;
            qb = a.B.codes + pb / 2;
            qsb = a.B.scales + pb / 32;
            const int ta = (int)(a.N - m0 < 256 ? a.N - m0 : 256) - 1;
            const uint32_t cs = (uint32_t)len / 2, ss = (uint32_t)len / 32;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int row = 32 * wave + 8 * v + (l >> 3);
                const uint32_t seg = seg0 ^ (64u * (v & 1));
                va[v] = (uint32_t)(row < ta ? row : ta) * cs + seg;
                vb[v] = (uint32_t)(row < tb ? row : tb) * cs + seg;
            }
            wsa = (uint32_t)(rs < ta ? rs : ta) * ss + 4u * (l & 1);
            wsb = (uint32_t)(rs < tb ? rs : tb) * ss + 4u * (l & 1);
        } else {
            const int64_t w0 = (int64_t)e * a.N + n0;
            const uint32_t cs = (uint32_t)(a.K / 2);
            lcnt = (int)((a.K + 255) >> 8);
            qa = a.A.codes;
            qsa = a.A.scales;
            qb = a.B.codes + w0 * cs;
            qsb = a.B.scales + w0 * a.bscales;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int row = 32 * wave + 8 * v + (l >> 3);
                const uint32_t seg = seg0 ^ (64u * (v & 1));
                const uint32_t r = (uint32_t)row_next[v] < (uint32_t)a.arows ? (uint32_t)row_next[v] : (uint32_t)a.arows - 1u;
                va[v] = r * a.astride + seg;
                vb[v] = (uint32_t)(row < tb ? row : tb) * cs + seg;
            }
            const uint32_t r = (uint32_t)row_next[4] < (uint32_t)a.arows ? (uint32_t)row_next[4] : (uint32_t)a.arows - 1u;
            wsa = r * (a.astride >> 4) + 4u * (l & 1);
            wsb = (uint32_t)(rs < tb ? rs : tb) * a.bscales + 4u * (l & 1);
        }
        look_ahead(lpos + hop);
    };
    auto advance = [&]() GS_INLINE {                     // before the first transfer of a unit
        if (lcnt == 0) {
            lpos += hop;
            enter();
        }
        --lcnt;
        // B's codes end with the contraction: what lies behind is some other row's, or nobody's.  A's rows are padded, the gradient's
        // operands have room behind them.
        lblk = !WGRAD && lcnt == 0 ? (int)((a.K >> 5) - 8 * (((a.K + 255) >> 8) - 1)) : 8;
        qa = gs_uniform(qa);
        qb = gs_uniform(qb);
        qsa = gs_uniform(qsa);
        qsb = gs_uniform(qsb);
    };
    auto issue = [&](uint32_t buf, auto kc) GS_INLINE {
        constexpr int k = decltype(kc)::value;
        const uint32_t dc = lds0 + buf + 4096u * wave, ds = lds0 + buf + 256u * wave;
        if constexpr (k < 4) {
            gs_dma16<1024 * k>(dc, va[k], qa);
        } else if constexpr (k < 8) {
            uint32_t off = vb[k - 4];
            if constexpr (!WGRAD) {
                const int l = gs_fresh_lane();
                const uint32_t seg = (uint32_t)((l & 7) ^ (l >> 4)) ^ (4u * (k & 1));
                off -= (int)seg >= lblk ? 16u * seg : 0u;         // the row's first segment of the unit instead, unused
            }
            gs_dma16<MXS_CODES + 1024 * (k - 4)>(dc, off, qb);
        } else if constexpr (k == 8) {
            gs_dma4<2 * MXS_CODES>(ds, wsa, qsa);
        } else {
            gs_dma4<2 * MXS_CODES + MXS_SCALES>(ds, wsb, qsb);
        }
        if constexpr (k == MXS_DMA - 1) {
            qa += MX_KI / 2;
            qb += MX_KI / 2;
            qsa += MX_KI / 32;
            qsb += MX_KI / 32;
        }
    };

    look_ahead(start);
    enter();
    advance();
    gs_for<MXS_DMA>([&](auto k) GS_INLINE { issue(0, k); });
    advance();
    gs_for<MXS_DMA>([&](auto k) GS_INLINE { issue(MXS_UNIT, k); });

    float16_t acc[4][2];
    uvec4_t f[2][6];                                     // fragments of a step: 0 .. 3 of A's rows, 4 and 5 of B's
    uvec2_t raw[6];                                      // their rows' scale bytes of a unit
    uint32_t sx[6], sy[6];                               // steps 0 and 1, 2 and 3: bytes 0 and 2 are this lane's blocks
    uint32_t ad[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) ad[s] = 128u * li + 16u * (uint32_t)((2 * s + half) ^ (li >> 1 & 7));
    auto read_frag = [&](uint32_t bu, int s, int n, int x) GS_INLINE {
        const uint32_t at = (x < 4 ? 16384u * wa : MXS_CODES + 8192u * wb) + 4096u * (x & 3);
        f[n][x] = *reinterpret_cast<const uvec4_t*>(lds + bu + at + ad[s]);
    };
    auto read_scale = [&](uint32_t bu, int x) GS_INLINE {
        const uint32_t at = 2 * MXS_CODES + (x < 4 ? 1024u * wa : MXS_SCALES + 512u * wb) + 256u * (x & 3);
        raw[x] = *reinterpret_cast<const uvec2_t*>(lds + bu + at + 8u * li);
    };
    gs_meet<MXS_DMA>();
#pragma unroll
    for (int x = 0; x < 6; ++x) {
        read_frag(0, 0, 0, x);
        read_scale(0, x);
    }
#pragma unroll
    for (int x = 0; x < 6; ++x) sx[x] = raw[x].x >> (8 * half);
    mxs_settle_scales(sx);

    uint32_t b0 = 0;                                     // buffer of the unit in work
    // first: the accumulators start here; steps: of 64 elements, that this wave multiplies; last: of the tile, and its buffer takes the outputs
    auto unit = [&](auto first_, auto last_, int steps, bool only) GS_INLINE {
        constexpr bool first = decltype(first_)::value, last = decltype(last_)::value;
        const uint32_t b1 = MXS_UNIT - b0;
        gs_for<4>([&](auto sc_) GS_INLINE {
            constexpr int s = decltype(sc_)::value, n = s & 1;
            gs_for<8>([&](auto mc) GS_INLINE {
                constexpr int m = decltype(mc)::value, i = m & 3, j = m >> 2;
                if constexpr (s == 0 && m < 6) sy[m] = raw[m].y >> (8 * half);
                if constexpr (s < 3 && m < 6) read_frag(b0, s + 1, n ^ 1, m);
                if constexpr (s == 3) {
                    // the next unit is there, and this one's buffer has been read by all
                    if constexpr (m == 1) {
                        gs_meet<0>();
                        if constexpr (!last)
                            if (!first || !only) advance();
                    }
                    if constexpr (m >= 1 && m < 7) {
                        read_frag(b1, 0, 0, m - 1);
                        read_scale(b1, m - 1);
                    }
                    if constexpr (!last && m >= 1) {
                        if (!first || !only) {
                            issue(b0, std::integral_constant<int, m - 1>{});
                            if constexpr (m >= 5) issue(b0, std::integral_constant<int, m + 2>{});
                        }
                    }
                }
                const uint32_t as = s < 2 ? sx[i] : sy[i], bs = s < 2 ? sx[4 + j] : sy[4 + j];
                if ((first && s == 0) || s < steps) {
                    if constexpr (LINES) mxs_mfma<first && s == 0, n == 1>(acc[i][j], f[n][4 + j], f[n][i], bs, as);
                    else mxs_mfma<first && s == 0, n == 1>(acc[i][j], f[n][i], f[n][4 + j], as, bs);
                }
                __builtin_amdgcn_sched_barrier(0);
            });
        });
#pragma unroll
        for (int x = 0; x < 6; ++x) sx[x] = raw[x].x >> (8 * half);
        mxs_settle_scales(sx);
        b0 = b1;
    };
    int pos = start, exp = 0;
    for (;;) {
        int m0, n0;
        tile_of(pos, exp, m0, n0);
        const int64_t base = WGRAD ? (int64_t)exp * a.N : (int64_t)begin_of(exp), rows = WGRAD ? a.N : (int64_t)count_of(exp);
        const int64_t con = WGRAD ? (int64_t)count_of(exp) : a.K;
        const int niter = (int)((con + 255) >> 8);
        const bool busy = m0 + 128 * wa < rows;
        const int whole = busy ? 4 : 0, rest = busy ? (int)((con - 256 * (int64_t)(niter - 1) + 63) >> 6) : 0;
        unit(std::true_type{}, std::false_type{}, niter == 1 ? rest : whole, niter == 1);
        if (niter > 1) {
#pragma unroll 1
            for (int u = 2; u < niter; ++u) unit(std::false_type{}, std::false_type{}, whole, false);
            unit(std::false_type{}, std::true_type{}, rest, false);
        }
        const uint32_t bl = MXS_UNIT - b0;               // the last unit's buffer
#pragma unroll
        for (int i = 0; i < 4; ++i) mxs_settle(acc[i]);
        if (busy) {
            const int64_t N = WGRAD ? a.K : a.N;
            mx_store_wave<OUT, LINES, 4, 2>(acc, lds + bl + wave * mx_wave_rows<OUT, 2>(), C + base * ldc, ldc, m0 + 128 * wa, n0 + 64 * wb, rows,
                                            N, vec, mx_whole<LINES>(m0 + 128 * wa + 128 <= rows && n0 + 64 * wb + 64 <= N, vec), gs_fresh_lane());
        }
        pos += hop;
        if (pos >= total) break;
        // every wave has its rows out of the buffer before any transfers into it
        gs_meet<63>();
        advance();
        gs_for<MXS_DMA>([&](auto k) GS_INLINE { issue(bl, k); });
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // no transfer may outlive the workgroup's LDS
}
