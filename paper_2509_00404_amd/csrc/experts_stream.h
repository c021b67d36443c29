// The experts' products for many slots: one stream of units over ragged tiles (included by experts.hip, inside its namespace).
#pragma once

// The tiles and units are those of the dense MXFP4 stream: 256 x 256 outputs by 8 waves of 128 x 64, a unit of 256 contraction elements
// of both operands goes straight into one of two LDS buffers while the other is multiplied, and the next tile's units travel while this
// one ends.  What is different is where tiles lie and how long they are, which the device alone knows:
//   EX_PRODUCT  C[s, n]: the expert's slots against its N outputs; its last tile of slots is short.  The first operand's rows are the
//               slots', or the tokens' by way of token[]: those of the next tile are fetched while this one is multiplied.
//   EX_PARTS    EX_PRODUCT with the contraction cut into parts of part_units units, a tile for each: fp32 sums of part p go to rows p S and on
//               of C, and k_experts_join adds them up.  For products whose tiles are fewer than half the chip.
//   EX_WGRAD    dW_e[n, k] over the expert's slots: every tile whole, the contraction as long as the expert has slots.
// A workgroup works its way through the tiles, gridDim.x apart.  Neighbouring tiles are of one expert, up to EX_BAND of its column tiles wide,
// and every XCD works on a run of them: they share panels of both operands in its L2.
// Outputs are not read again here and go past the caches: kept in L2 they drive out the operands' panels (gradients of 8192 tokens' four
// experts, 2048 x 4096 each, 529 us with the quantizers, so 378; 16384 tokens' product 409, 401).  Gradients whose rows do not start on
// cache lines stay in L2, where the parts of a line meet (1384 x 2456 each, 403 tokens' five of 64 experts 152, past it 246; products,
// which write less, are 3 % better past it all the same).
// What bounds it: 16384 tokens' four experts, 2048 x 4096 each, 320 us (1.1 PFLOP, 3.4 PFLOP/s; an eighth of the tiles' rows is short tiles').
// Without its transfers it takes 250, without its matrix instructions 250, without its stores 285: LDS takes a unit's 192 KB of
// fragments and 68 KB of transfers while the matrix pipe has 2048 cycles of work.  The matrix pipe is busy 0.48 of the clocks (1.8 GHz held), LDS
// reads 0.27, and the waves wait 0.39 of their time where units meet; at 60 rows an expert 0.23, 0.22 and 0.57.  Gradients of 8192 tokens' (1.07 GB out) 285 to 320, without
// stores 165.  Tried: tiles of 32 rows fewer to multiply at a short tile's end, transfers left out there, bands of 4 and 16, no XCD order: 1 % up
// or down; whole tiles of all experts before the short ones: 3 % slower, 4 % faster at 60 rows an expert; a lane's own 32-byte stores instead
// of lines by way of LDS: 391 for 362 with the quantizers, gradients 546 for 378.
// A wave whose 128 rows lie behind the tile's end multiplies nothing, and a last unit that exists in part is multiplied by steps of 64.
#define EX_BAND 8
enum { EX_PRODUCT = 0, EX_WGRAD = 1, EX_PARTS = 2 };
struct ExStream {
    MxRows A, B;                          // first operand (slots, or N), second (weights, or K)
    const int32_t* offsets;
    const int32_t* token;                 // null: rows by slot
    int64_t S, arows;                     // slots; rows of A
    int64_t N;                            // product: outputs of an expert; gradient: N
    int64_t K;                            // product: contraction, a multiple of 32; gradient: K
    uint32_t astride;                     // product: bytes of a row of A's codes, a multiple of 128 (its tail is zeros)
    int64_t ascales, bscales;             // from one unit's scales to the next one's
    int E, tiles_m, tiles_n;              // gradient: tiles_m along N, tiles_n along K; product: tiles_n along N
    int parts, part_units;                // EX_PARTS: the parts, none of them empty, and the units of each but the last
};
// Behind the two buffers a wave has room to turn 16 rows of its outputs into whole lines, every expert has two numbers, and the workgroup
// its next tiles.
#define EX_STAGE_ROW 144                                 // 64 bf16 and 16 bytes that spread the rows over the banks
#define EX_STAGE (16 * EX_STAGE_ROW)
#define EX_HALF 48                                       // tiles that are looked up at a time
#define EX_LIST (MXS_LDS + 8 * EX_STAGE + 2 * 4 * (EXPERTS_MAX + 1) + 8)
#define EX_LDS (EX_LIST + 2 * EX_HALF * 16)
static_assert(EX_LIST % 16 == 0 && EX_LDS <= 160 * 1024, "fits a CU");

// gs_meet with `stores` younger stores on their way, rounded down to an even number
__device__ __forceinline__ void ex_meet(int stores) {
    switch (stores >> 1) {
        case 8: gs_meet<16>(); break;
        case 7: gs_meet<14>(); break;
        case 6: gs_meet<12>(); break;
        case 5: gs_meet<10>(); break;
        case 4: gs_meet<8>(); break;
        case 3: gs_meet<6>(); break;
        case 2: gs_meet<4>(); break;
        case 1: gs_meet<2>(); break;
        default: gs_meet<0>(); break;
    }
}
// zeros to n elements from p
template <typename OUT>
__device__ __forceinline__ void ex_clear(OUT* p, int64_t n, bool vec) {
    constexpr int E = 16 / (int)sizeof(OUT);
    const int64_t units = vec ? n / E : 0;
    for (int64_t c = threadIdx.x; c < units; c += 512) reinterpret_cast<uvec4_t*>(p)[c] = uvec4_t{0u, 0u, 0u, 0u};
    for (int64_t c = units * E + threadIdx.x; c < n; c += 512) p[c] = OUT(0);
}

// A wave's accumulator tiles (transposed, bf16) to memory: 16 rows of its 64 columns at a time are staged at sm, eight lanes a row.
// A store for every eight rows: 16 where all are there.
template <bool PAST>
__device__ __forceinline__ void ex_store_lines(const float16_t (&acc)[4][2], uint8_t* sm, bf16_t* __restrict__ C, int64_t ldc, int64_t m0, int64_t n0,
                                               int64_t M, int64_t N, bool vec, bool whole, int lane) {
    const int li = lane & 31, half = lane >> 5, unit = lane & 7;
    const int64_t c = n0 + 8 * unit;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if ((li >> 4) == h) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int v = 0; v < 16; v += 4)
                        mx_put4(reinterpret_cast<bf16_t*>(sm + (li & 15) * EX_STAGE_ROW) + 32 * j + 2 * v + 4 * half, acc[i][j][v],
                                acc[i][j][v + 1], acc[i][j][v + 2], acc[i][j][v + 3]);
            }
            gs_wave_order();
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int row = 8 * t + (lane >> 3);
                const uint8_t* q = sm + row * EX_STAGE_ROW + 16 * unit;
                const int64_t r = m0 + 32 * i + 16 * h + row, left = N - c;
                if (!whole && r - (lane >> 3) >= M) continue;             // (for the whole wave)
                bf16_t* p = C + r * ldc + c;
                if (whole || (r < M && vec && left >= 8)) {
                    const uvec4_t w = *reinterpret_cast<const uvec4_t*>(q);
                    if constexpr (PAST) __builtin_nontemporal_store(w, reinterpret_cast<uvec4_t*>(p));
                    else *reinterpret_cast<uvec4_t*>(p) = w;
                } else if (r < M) {
#pragma unroll 1
                    for (int e = 0; e < 8 && e < left; ++e) p[e] = reinterpret_cast<const bf16_t*>(q)[e];
                }
            }
            gs_wave_order();
        }
}

// fp32: a row of 32 is a whole line as it is
template <bool PAST>
__device__ __forceinline__ void ex_store_plain(const float16_t (&acc)[4][2], float* __restrict__ C, int64_t ldc, int64_t m0, int64_t n0, int64_t M,
                                               int64_t N, bool whole, int lane) {
    const int64_t c = n0 + (lane & 31), row = 4 * (lane >> 5);
    const int rows = M - m0 < 128 ? (int)(M - m0) : 128, cols = N - c < 64 ? (int)(N - c) : 64;
    float* p = C + (m0 + row) * ldc + c;                 // the lane's first; the next of its rows, the fifth one 8 behind the first
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const bool there = whole || 32 * i + (int)row + 8 * (v >> 2) + (v & 3) < rows;
            if constexpr (PAST) {
                if (there && (whole || 0 < cols)) __builtin_nontemporal_store(acc[i][0][v], p);
                if (there && (whole || 32 < cols)) __builtin_nontemporal_store(acc[i][1][v], p + 32);
            } else {
                if (there && (whole || 0 < cols)) p[0] = acc[i][0][v];
                if (there && (whole || 32 < cols)) p[32] = acc[i][1][v];
            }
            p += v % 4 == 3 ? 5 * ldc : ldc;
        }
}

// a tile: its expert, its first row in the expert and column, and the expert's first slot (product) or slots (gradient), or its part
struct __attribute__((aligned(16))) ExTile {
    int expert, m0, n0, at;
};

// PAST: outputs go past the caches
template <typename OUT, int MODE, bool PAST>
__global__ void __launch_bounds__(512, 2)
k_experts_stream(ExStream a, OUT* __restrict__ C, int64_t ldc, bool vec) {
    constexpr bool LINES = sizeof(OUT) == 2;             // outputs by way of LDS, accumulator tiles transposed
    constexpr bool WGRAD = MODE == EX_WGRAD, PARTS = MODE == EX_PARTS;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    uint8_t* const s_stage = lds + MXS_LDS;
    int32_t* const s_begin = reinterpret_cast<int32_t*>(s_stage + 8 * EX_STAGE);     // an expert's first slot, and the end of all
    // product: the first tile of every expert, and their number.  Gradient: the experts with slots before it (low 10 bits; their number)
    // and above these the segments of SLOT_ALIGN before it
    int32_t* const s_first = s_begin + EXPERTS_MAX + 1;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wa = wave >> 2, wb = wave & 3;
    const int lane = (int)threadIdx.x & 63, li = lane & 31, half = lane >> 5;

    // ---- the tables, by every expert's thread
    {
        const int e = (int)threadIdx.x;
        int32_t* s_sum = reinterpret_cast<int32_t*>(lds);                            // (the waves' sums, before any unit is here)
        // offsets held to 0 .. S and to ascend, whatever the memory says
        int32_t b = e < a.E ? (int32_t)held(a.offsets[e], a.S) : 0, all = (int32_t)held(a.offsets[a.E], a.S);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int32_t o = __shfl_up(b, d);
            if (lane >= d && o > b) b = o;
        }
        if (lane == 63) s_sum[wave] = b;
        __syncthreads();
        for (int w = 0; w < wave; ++w) b = b > s_sum[w] ? b : s_sum[w];
        if (e < a.E) s_begin[e] = b;
        if (e == a.E - 1) s_begin[a.E] = all > b ? all : b;
        __syncthreads();
        const int32_t n = e < a.E ? s_begin[e + 1] - b : 0;
        int32_t mine = WGRAD ? (n > 0) | (n + SLOT_ALIGN - 1) / SLOT_ALIGN << 10 : ((n + 255) >> 8) * a.tiles_n * (PARTS ? a.parts : 1), upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int32_t o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        if (lane == 63) s_sum[8 + wave] = upto;
        __syncthreads();
        for (int w = 0; w < wave; ++w) upto += s_sum[8 + w];
        if (e < a.E) s_first[e] = upto - mine;
        if (e == a.E - 1) s_first[a.E] = upto;
        __syncthreads();
    }
    auto table = [&](const int32_t* t, int e) GS_INLINE { return __builtin_amdgcn_readfirstlane(t[e]); };
    auto begin_of = [&](int e) GS_INLINE { return table(s_begin, e); };
    auto count_of = [&](int e) GS_INLINE { return table(s_begin, e + 1) - table(s_begin, e); };
    auto first_of = [&](int e) GS_INLINE { return WGRAD ? (table(s_first, e) & 1023) * (a.tiles_m * a.tiles_n) : table(s_first, e); };
    const int total = first_of(a.E);

    // ---- what no tile covers
    if constexpr (WGRAD) {
        for (int e = 0; e < a.E; ++e)                                                // experts without slots
            if (count_of(e) == 0)
                for (int64_t r = blockIdx.x; r < a.N; r += gridDim.x) ex_clear(C + ((int64_t)e * a.N + r) * ldc, a.K, vec);
    } else if constexpr (!PARTS) {
        for (int64_t r = (int64_t)begin_of(a.E) + blockIdx.x; r < a.S; r += gridDim.x)      // slots that serve no choice
            ex_clear(C + r * ldc, a.N, vec);
    }

    // ---- this workgroup's tiles.  A tile's place takes a search and two divisions, some thousand cycles one after the other: 48 lanes do them
    // for 48 tiles at once, a half of a ring ahead.  (Done by every wave for every tile, 1664 tiles of a single unit took 37 us without any
    // transfer or store; 533 tokens' gradients, 128 experts of 80 x 3240, 90 us instead of 67.)
    const int hop = (int)gridDim.x, xcds = (hop & 7) == 0 ? 8 : 1;
    const int start = ((int)blockIdx.x % xcds) * (hop / xcds) + (int)blockIdx.x / xcds;
    if (start >= total) return;
    const int tiles = (total - start + hop - 1) / hop;
    ExTile* const s_list = reinterpret_cast<ExTile*>(lds + EX_LIST);
    auto fill = [&](int half_no) GS_INLINE {
        const int i = (int)threadIdx.x, t = half_no * EX_HALF + i;
        if (i >= EX_HALF || t >= tiles) return;
        const int tile = start + t * hop, per = a.tiles_m * a.tiles_n;
        auto first = [&](int e) GS_INLINE { return WGRAD ? (s_first[e] & 1023) * per : s_first[e]; };
        int lo = 0, hi = a.E;                            // first(lo) <= tile < first(hi)
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first(mid) <= tile) lo = mid;
            else hi = mid;
        }
        const int count = s_begin[lo + 1] - s_begin[lo], down = WGRAD ? a.tiles_m : (count + 255) >> 8;
        int local = tile - first(lo), part = 0;
        if constexpr (PARTS) {
            part = local / (down * a.tiles_n);
            local -= part * (down * a.tiles_n);
        }
        const int band = local / (EX_BAND * down), r = local - band * EX_BAND * down;
        const int left = a.tiles_n - band * EX_BAND, w = left < EX_BAND ? left : EX_BAND, tm = r / w;
        s_list[t % (2 * EX_HALF)] = {lo, 256 * tm, 256 * (band * EX_BAND + r - tm * w), WGRAD ? count : PARTS ? part : s_begin[lo]};
    };
    fill(0);
    fill(1);
    __syncthreads();
    auto tile_at = [&](int t) GS_INLINE {
        const uvec4_t v = *reinterpret_cast<const uvec4_t*>(s_list + t % (2 * EX_HALF));
        return ExTile{__builtin_amdgcn_readfirstlane((int)v[0]), __builtin_amdgcn_readfirstlane((int)v[1]),
                      __builtin_amdgcn_readfirstlane((int)v[2]), __builtin_amdgcn_readfirstlane((int)v[3])};
    };

    auto slots_at = [&](const ExTile& t) GS_INLINE { return PARTS ? begin_of(t.expert) : t.at; };

    // ---- transfers
    const uint8_t *qa, *qb, *qsa, *qsb;                  // the next unit's codes, and this wave's part of its scales
    int ltile = 0, lcnt = 0, lblk = 8;                   // tile being fetched, units left of it, blocks of 32 of the unit that B has
    bool lends = true;                                   // whether its last unit is the contraction's
    uint32_t va[4], vb[4];                               // the lane's offsets
    int32_t row_next[4];                                 // rows of A of the tile to be entered next, by this lane's place
    ExTile next;                                         // that tile
    auto look_ahead = [&](int t) GS_INLINE {
        next = tile_at(t < tiles ? t : tiles - 1);       // (past the end: the last one again, unused)
        if constexpr (!WGRAD) {
            const int l = gs_fresh_lane();
            const int32_t b = slots_at(next) + next.m0, last = begin_of(next.expert + 1) - b - 1;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int row = 32 * wave + 8 * v + (l >> 3);
                row_next[v] = b + (row < last ? row : last);
                if (a.token) row_next[v] = a.token[row_next[v]];
            }
        }
    };
    auto enter = [&]() GS_INLINE {
        const int e = next.expert, m0 = next.m0, n0 = next.n0;
        const int l = gs_fresh_lane();
        const uint32_t seg0 = (uint32_t)((l & 7) ^ (l >> 4)) * 16;
        const int64_t brows = WGRAD ? a.K : a.N;
        const int tb = (int)(brows - n0 < 256 ? brows - n0 : 256) - 1;
        if constexpr (WGRAD) {
            const int units = (next.at + SLOT_ALIGN - 1) / SLOT_ALIGN, len = units * SLOT_ALIGN;
            const int64_t at = (int64_t)(table(s_first, e) >> 10) * SLOT_ALIGN;
            const int64_t pa = at * a.N + (int64_t)m0 * len, pb = at * a.K + (int64_t)n0 * len;
            lcnt = units;
            qa = a.A.codes + pa / 2;
            qsa = a.A.scales + at * a.N / 32 + 8 * (m0 + 32 * wave);
            qb = a.B.codes + pb / 2;
            qsb = a.B.scales + at * a.K / 32 + 8 * (n0 + 32 * wave);
            const int ta = (int)(a.N - m0 < 256 ? a.N - m0 : 256) - 1;
            const uint32_t cs = (uint32_t)len / 2;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int row = 32 * wave + 8 * v + (l >> 3);
                const uint32_t seg = seg0 ^ (64u * (v & 1));
                va[v] = (uint32_t)(row < ta ? row : ta) * cs + seg;
                vb[v] = (uint32_t)(row < tb ? row : tb) * cs + seg;
            }
        } else {
            const int64_t w0 = (int64_t)e * a.N + n0;
            const uint32_t cs = (uint32_t)(a.K / 2);
            lcnt = (int)((a.K + 255) >> 8);
            qa = a.A.codes;
            qsa = a.A.scales + 8 * (int64_t)(slots_at(next) + m0 + 32 * wave);
            qb = a.B.codes + w0 * cs;
            qsb = a.B.scales + 8 * (w0 + 32 * wave);
            if constexpr (PARTS) {
                const int u0 = next.at * a.part_units, left = lcnt - u0;
                lends = left <= a.part_units;
                lcnt = lends ? left : a.part_units;
                qa += (int64_t)u0 * (MX_KI / 2);
                qb += (int64_t)u0 * (MX_KI / 2);
                qsa += u0 * a.ascales;
                qsb += u0 * a.bscales;
            }
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int row = 32 * wave + 8 * v + (l >> 3);
                const uint32_t seg = seg0 ^ (64u * (v & 1));
                const uint32_t r = (uint32_t)row_next[v] < (uint32_t)a.arows ? (uint32_t)row_next[v] : (uint32_t)a.arows - 1u;
                va[v] = r * a.astride + seg;
                vb[v] = (uint32_t)(row < tb ? row : tb) * cs + seg;
            }
        }
        look_ahead(++ltile);
    };
    auto advance = [&]() GS_INLINE {                     // before the first transfer of a unit
        if (lcnt == 0) enter();
        --lcnt;
        // B's codes end with the contraction: what lies behind is some other row's, or nobody's.  A's rows are padded, the gradient's
        // operands have room behind them.
        lblk = !WGRAD && lcnt == 0 && lends ? (int)((a.K >> 5) - 8 * (((a.K + 255) >> 8) - 1)) : 8;
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
            gs_dma4<2 * MXS_CODES>(ds, 4u * gs_fresh_lane(), qsa);
        } else {
            gs_dma4<2 * MXS_CODES + MXS_SCALES>(ds, 4u * gs_fresh_lane(), qsb);
        }
        if constexpr (k == MXS_DMA - 1) {
            qa += MX_KI / 2;
            qb += MX_KI / 2;
            qsa += a.ascales;
            qsb += a.bscales;
        }
    };

    look_ahead(0);
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
    // first: the accumulators start here; steps: of 64 elements, that this wave multiplies.  kept: the last tile's stores, which are younger than the
    // transfers that the unit waits for and may stay on their way.
    auto unit = [&](auto first_, int steps, int kept) GS_INLINE {
        constexpr bool first = decltype(first_)::value;
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
                        if constexpr (first) ex_meet(kept);
                        else gs_meet<0>();
                        advance();
                    }
                    if constexpr (m >= 1 && m < 7) {
                        read_frag(b1, 0, 0, m - 1);
                        read_scale(b1, m - 1);
                    }
                    if constexpr (m >= 1) {
                        issue(b0, std::integral_constant<int, m - 1>{});
                        if constexpr (m >= 5) issue(b0, std::integral_constant<int, m + 2>{});
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
    int kept = 0;
#pragma unroll 1
    for (int t = 0; t < tiles; ++t) {
        // the half of the ring that the tiles before have left, which no wave reads any more
        if (t > EX_HALF && t % EX_HALF == 1) fill(t / EX_HALF + 1);
        const ExTile now = tile_at(t);
        const int64_t base = WGRAD ? (int64_t)now.expert * a.N : (int64_t)slots_at(now) + (PARTS ? now.at * a.S : 0);
        const int64_t rows = WGRAD ? a.N : (int64_t)(begin_of(now.expert + 1) - slots_at(now));
        int64_t con = WGRAD ? (int64_t)now.at : a.K;
        if constexpr (PARTS) {
            const int64_t long_ = 256 * (int64_t)a.part_units;
            con -= now.at * long_;
            con = con < long_ ? con : long_;
        }
        const int niter = (int)((con + 255) >> 8);
        const int64_t r = now.m0 + 128 * wa, c = now.n0 + 64 * wb, N = WGRAD ? a.K : a.N;
        const bool busy = r < rows && c < N;
        const int whole = busy ? 4 : 0, rest = busy ? (int)((con - 256 * (int64_t)(niter - 1) + 63) >> 6) : 0;
        unit(std::true_type{}, niter == 1 ? rest : whole, kept);
#pragma unroll 1
        for (int u = 1; u < niter; ++u) unit(std::false_type{}, u == niter - 1 ? rest : whole, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) mxs_settle(acc[i]);
        kept = 0;
        if (busy) {
            const bool inside = r + 128 <= rows && c + 64 <= N;
            if constexpr (LINES) {
                ex_store_lines<PAST>(acc, s_stage + wave * EX_STAGE, C + base * ldc, ldc, r, c, rows, N, vec, inside && vec, gs_fresh_lane());
                // one store for every eight rows there are, where no row's end is stored piece by piece
                if (vec && N % 8 == 0) kept = inside ? 16 : rows - r < 128 ? (int)((rows - r + 7) >> 3) : 16;
            } else {
                ex_store_plain<PAST>(acc, C + base * ldc, ldc, r, c, rows, N, inside, gs_fresh_lane());
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // no transfer may outlive the workgroup's LDS
}
