// Forward of a batch over a 4-bit weight where reading the weight back first would cost more than decoding it in the product:
//   y = g (.) (x W^T + s h B^T) (+ bias), h = x A^T there already, rounded once to the storage type: it is the operand of a 16-bit
// product, and the tensor that a backward is given.
//
// A workgroup owns a tile of rows of W and of tokens.  Steps of 128 columns go through three LDS stages filled by direct loads
// (codes as they are, a quarter of the bytes of a 16-bit weight; x in 16 bits), the low-rank part through the same stages, 64 ranks
// at a time, first.  A wave decodes the codes of its rows once and multiplies them with the fragments of its tokens.  Products are
// summed in fp32 within a group and the sum is multiplied by the scale in fp32, as in the streaming kernel: no weight is rounded.
// A zero point that is the same everywhere enters as the MFMA's addend, -8 times the sum of x that one MFMA against a constant
// gives for all rows.
//
// Bound: reading the codes up to about 64 tokens, beyond by issuing: a wave's 80 MFMAs of a step (16 of them for the sums of x) and the
// 300 vector instructions of decoding and scaling its rows share one port.  A forward with weights from memory: 8192 x 8192, r 64, 256
// tokens 80 us (92 with the weight read back first), 14336 x 4096, 64 tokens 41 us (64).
#include "quant_codes.hpp"

namespace dora {
namespace {

// WR x WT waves, each with MR blocks of 16 rows of W and TB blocks of 16 tokens; SUB: k-steps of 32 to a scale; ZERO: zero points
template <int WR, int WT, int MR, int TB, int CODE, int SUB, bool ZERO, int DT>
__global__ __launch_bounds__(64 * WR * WT) void quant_tile_kernel(QuantTileArgs p)
{
    typedef Elem16<DT> E;
    constexpr bool INT = CODE == DORA_QUANT_INT4;
    constexpr int WAVES = WR * WT, THREADS = 64 * WAVES, ROWS = WR * MR * 16, TOK = WT * TB * 16, STAGES = 3;
    constexpr int W_BYTES = ROWS * 64, X_BYTES = TOK * 256, STAGE = W_BYTES + X_BYTES;
    constexpr int WL = W_BYTES / 1024 / WAVES, XL = X_BYTES / 1024 / WAVES, LPS = WL + XL;   // loads of a wave for a stage
    static_assert(WL * WAVES * 1024 == W_BYTES && XL * WAVES * 1024 == X_BYTES && XL % 2 == 0, "loads of a stage");
    static_assert(2 * W_BYTES + X_BYTES / 2 == STAGE, "64 ranks of B and h take a stage");
    static_assert(THREADS == 2 * ROWS, "a wave to 64 rows of scales and one to 64 rows of zero points");
    constexpr int PIECE = 8, SCALES = ROWS * PIECE * 2;   // groups whose scales come in one go, their bytes; the zero points follow
    constexpr int RED_LD = ROWS + 4;
    constexpr int TOP = STAGES * STAGE + 2 * 2 * SCALES, RED = TOK * RED_LD * 4;
    __shared__ __attribute__((aligned(1024))) char smem[TOP > RED ? TOP : RED];
    static_assert(sizeof(smem) <= 160 * 1024, "LDS of a gfx950 CU");

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, lq = lane >> 4, wr = wave / WT, wt = wave % WT;
    const int T = p.T, N = p.w.d_out, K = p.w.d_in, r = p.r;
    // consecutive ids go to the XCDs in turn: undone, so that the token tiles and slices of the same rows share an L2
    const int total_wg = (int)gridDim.x, id = (int)blockIdx.x, xcd = id & 7, xq = total_wg >> 3, xr = total_wg & 7;
    const int logical = (xcd < xr ? xcd * (xq + 1) : xr * (xq + 1) + (xcd - xr) * xq) + (id >> 3);
    const int z = logical % p.ksplit, tile = logical / p.ksplit;
    const int t0 = tile % p.token_tiles * TOK, n0 = tile / p.token_tiles * ROWS;
    const int rows = N - n0 < ROWS ? N - n0 : ROWS, toks = T - t0 < TOK ? T - t0 : TOK;
    const uint32_t smem_lds = (uint32_t)(uintptr_t)(lds_cptr_t)smem, scales_lds = smem_lds + STAGES * STAGE;

    // steps of this slice: the low-rank part in the first one, whole steps of columns, what the rows end in behind the last one's
    const int whole = K / BLOCK_K, blocks = (K + BLOCK_K - 1) / BLOCK_K;
    const int k_first = (int)((int64_t)whole * z / p.ksplit), k_end = (int)((int64_t)whole * (z + 1) / p.ksplit);
    const int low = z == 0 ? (r + 63) / 64 : 0, steps = low + k_end - k_first;

    const uint32_t row_bytes = (uint32_t)K / 2;
    __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint32_t*>(p.w.q + (int64_t)n0 * (K / 8)), 0,
                                                                  (int)(uint32_t)((int64_t)rows * row_bytes), 0x00020000);
    __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(p.x + (int64_t)t0 * K), 0,
                                                                  (int)(uint32_t)((int64_t)toks * K * 2), 0x00020000);
    __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(p.b + (int64_t)n0 * r), 0,
                                                                  (int)(uint32_t)((int64_t)rows * r * 2), 0x00020000);
    __amdgpu_buffer_rsrc_t rh = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(p.h + (int64_t)t0 * r), 0,
                                                                  (int)(uint32_t)((int64_t)toks * r * 2), 0x00020000);
    // A stage in chunks of 16 bytes, swizzled so that the sixteen rows of a fragment lie in different banks: rows of W of 64 bytes,
    // then of x of 256 (low-rank steps: of B and of h, 128 bytes each).  Row and chunk travel in the vector offset, which alone is
    // range checked, the step in the scalar one.
    uint32_t vw[WL], vx[XL], vb[2 * WL], vh[XL / 2];
    int kb[2 * WL], kh[XL / 2];
#pragma unroll
    for (int i = 0; i < WL; ++i) {
        const int row = (wave * WL + i) * 16 + (lane >> 2);
        vw[i] = row < rows ? (uint32_t)row * row_bytes + (uint32_t)((lane & 3) ^ ((row >> 2) & 3)) * 16u : OUTSIDE;
    }
#pragma unroll
    for (int i = 0; i < XL; ++i) {
        const int row = (wave * XL + i) * 4 + (lane >> 4);
        vx[i] = row < toks ? (uint32_t)row * (uint32_t)K * 2u + (uint32_t)((lane & 15) ^ (row & 15)) * 16u : OUTSIDE;
    }
#pragma unroll
    for (int i = 0; i < 2 * WL; ++i) {
        const int row = (wave * 2 * WL + i) * 8 + (lane >> 3);
        kb[i] = ((lane & 7) ^ ((row >> 1) & 7)) * 8;
        vb[i] = row < rows ? ((uint32_t)row * (uint32_t)r + (uint32_t)kb[i]) * 2u : OUTSIDE;
    }
#pragma unroll
    for (int i = 0; i < XL / 2; ++i) {
        const int row = (wave * (XL / 2) + i) * 8 + (lane >> 3);
        kh[i] = ((lane & 7) ^ ((row >> 1) & 7)) * 8;
        vh[i] = row < toks ? ((uint32_t)row * (uint32_t)r + (uint32_t)kh[i]) * 2u : OUTSIDE;
    }
    // load I of a step of columns into a stage (zeros past the last step)
    auto issue_one = [&](auto i_tag, int step, int stage) {
        constexpr int I = decltype(i_tag)::value;
        char* const at = smem + stage * STAGE;
        const bool in = step < steps;
        const uint32_t k0 = in ? (uint32_t)(k_first + step - low) * BLOCK_K : 0u;
        if constexpr (I < WL) load_1k(at + (wave * WL + I) * 1024, rw, in ? vw[I] : OUTSIDE, k0 / 2);
        else load_1k(at + W_BYTES + (wave * XL + I - WL) * 1024, rx, in ? vx[I - WL] : OUTSIDE, k0 * 2);
    };
    // the loads of a step, as many whatever it is
    auto issue = [&](int step, int stage) {
        char* const at = smem + stage * STAGE;
        if (step < low) {
            const int l0 = step * 64;
#pragma unroll
            for (int i = 0; i < 2 * WL; ++i) load_1k(at + (wave * 2 * WL + i) * 1024, rb, l0 + kb[i] < r ? vb[i] : OUTSIDE, (uint32_t)l0 * 2u);
#pragma unroll
            for (int i = 0; i < XL / 2; ++i)
                load_1k(at + 2 * W_BYTES + (wave * (XL / 2) + i) * 1024, rh, l0 + kh[i] < r ? vh[i] : OUTSIDE, (uint32_t)l0 * 2u);
        } else {
            static_for<LPS>([&](auto i) { issue_one(i, step, stage); });
        }
    };
    const uint32_t rs_at = (uint32_t)((wr * MR * 16 + l16) * (PIECE * 2));
    // Scales (the first half of the waves) and zero points of eight groups at a time, a row to a lane, two steps ahead of their use.
    // (A step's at a time every lane's 2 bytes are a line of their own to the L1, 512 of the 1300 cycles that a step's loads take.
    // Through registers the compiler waits for every load in flight before it uses them.)  The last piece ends with the row.
    const int s_row = (int)threadIdx.x % ROWS, s_half = wave / (WAVES / 2);
    const uint32_t scale_bytes = (uint32_t)p.w.groups * 2u;
    __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char*>(static_cast<const char*>(ZERO && s_half ? p.w.zero : p.w.scale) + (int64_t)n0 * scale_bytes), 0,
        (int)((uint32_t)rows * scale_bytes), 0x00020000);
    const uint32_t vs = s_row < rows ? (uint32_t)s_row * scale_bytes : OUTSIDE;
    auto group_of = [&](int block) { return (int)(((int64_t)block * BLOCK_K) >> p.w.group_shift); };   // that a block of columns begins in
    auto piece_start = [&](int g) { return g / PIECE * PIECE < p.w.groups - PIECE ? g / PIECE * PIECE : p.w.groups - PIECE; };
    auto issue_piece = [&](int g) {
        load_1k(smem + STAGES * STAGE + (g / PIECE & 1) * (2 * SCALES) + s_half * SCALES + wave % (WAVES / 2) * 1024, rs, vs,
                (uint32_t)piece_start(g) * 2u);
    };
    // where block b's scales begin
    auto scales_at = [&](int b) {
        const int g = group_of(b);
        return scales_lds + (uint32_t)(g / PIECE & 1) * (2 * SCALES) + (uint32_t)(g - piece_start(g)) * 2u + rs_at;
    };

    f32x4_t acc[MR][TB];
#pragma unroll
    for (int i = 0; i < MR; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // LDS reads of a lane, relative to the stage.  A round is two k-steps, 64 columns (groups of 32: one); a lane's share of it is
    // consecutive columns: 8 bytes of codes (4).
    constexpr int KS = SUB == 1 ? 1 : 2, ROUNDS = 4 / KS;
    uint32_t rx_at[4], rw_at[ROUNDS], rl_at[2];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int chunk = SUB == 1 ? q * 4 + lq : q / 2 * 8 + lq * 2 + q % 2;
        rx_at[q] = (uint32_t)(W_BYTES + (wt * TB * 16 + l16) * 256 + (chunk ^ l16) * 16);
        const uint32_t row = (uint32_t)((wr * MR * 16 + l16) * 64);
        if constexpr (SUB == 1) rw_at[q] = row + (uint32_t)((q ^ (l16 >> 2)) * 16 + lq * 4);
        else if (q % 2 == 0) rw_at[q / 2] = row + (uint32_t)(((q + (lq >> 1)) ^ (l16 >> 2)) * 16 + (lq & 1) * 8);
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) rl_at[q] = (uint32_t)(l16 * 128 + (((q * 4 + lq) ^ (l16 >> 1)) & 7) * 16);
    const uint32_t addend = INT && !ZERO ? (DT == DT_BF16 ? 0xc100c100u : 0xc800c800u) : (DT == DT_BF16 ? 0x3f803f80u : 0x3c003c00u);   // -8, 1
    const bf16x8_t constant = __builtin_bit_cast(bf16x8_t, u32x4_t{addend, addend, addend, addend});

    // What a round needs, read a round ahead, in as many parts as the round before it has blocks of TB products: one behind each, as
    // a wave that asks for all of it in one go waits for the LDS before its first product (900 of 5600 cycles a step).
    constexpr int BLOCKS = MR * KS, XPART = KS * TB / BLOCKS;
    static_assert(XPART * BLOCKS == KS * TB && KS * TB >= BLOCKS, "parts of a round's reads");
    struct Round { bf16x8_t x[KS][TB]; uint32_t w[MR][KS], s[MR], z[MR]; };
    auto read_part = [&](auto h_tag, auto blk_tag, Round& q, uint32_t at, uint32_t sat) {
        constexpr int h = decltype(h_tag)::value, n = SUB == 4 ? 0 : h, blk = decltype(blk_tag)::value, i = blk / KS;
        if constexpr (blk % KS == 0) {
            if constexpr (SUB == 1) {
                q.w[i][0] = lds_read_b32<i * 1024>(at + rw_at[h]);
            } else {
                const uint64_t v = lds_read_b64<i * 1024>(at + rw_at[h]);
                q.w[i][0] = (uint32_t)v; q.w[i][KS - 1] = (uint32_t)(v >> 32);
            }
        }
        if constexpr (blk % KS == KS - 1) {
            q.s[i] = lds_read_u16<i * 16 * PIECE * 2 + n * 2>(sat);
            if constexpr (ZERO) q.z[i] = lds_read_u16<SCALES + i * 16 * PIECE * 2 + n * 2>(sat);
        }
        static_for<XPART>([&](auto it) {
            constexpr int e = blk * XPART + decltype(it)::value, u = e / TB, j = e % TB;
            q.x[u][j] = lds_read_b128<j * 4096>(at + rx_at[KS * h + u]);
        });
    };
    auto read = [&](auto h_tag, Round& q, uint32_t at, uint32_t sat) {
        static_for<BLOCKS>([&](auto blk) { read_part(h_tag, blk, q, at, sat); });
    };
    // behind: called after each block of products, with its number
    auto multiply = [&](const Round& q, auto&& behind) {
        f32x4_t first[TB];                             // what the products are added to: -8 (or 1) times the sum of x
#pragma unroll
        for (int u = 0; u < KS; ++u)
#pragma unroll
            for (int j = 0; j < TB; ++j)
                if constexpr (INT) first[j] = E::mfma16(q.x[u][j], constant, u == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : first[j]);
                else first[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        f32x4_t part[TB];
        static_for<BLOCKS>([&](auto blk_tag) {
            constexpr int blk = decltype(blk_tag)::value, i = blk / KS, u = blk % KS;
            if constexpr (u == 0) {
#pragma unroll
                for (int j = 0; j < TB; ++j) {
                    part[j] = first[j];
                    if constexpr (ZERO) {
                        const float zp = -E::lo(q.z[i]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) part[j][e] *= zp;
                    }
                }
            }
            const bf16x8_t wf = decode_fragment<CODE, DT>(q.w[i][u]);
#pragma unroll
            for (int j = 0; j < TB; ++j) part[j] = E::mfma16(q.x[u][j], wf, part[j]);
            behind(blk_tag);
            if constexpr (u == KS - 1) {
                const float s = E::lo(q.s[i]);
#pragma unroll
                for (int j = 0; j < TB; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(s, part[j][e], acc[i][j][e]);
            }
        });
    };
    auto multiply_low = [&](uint32_t at) {
        bf16x8_t hf[2][TB], bf[2][MR];
        static_for<2 * TB>([&](auto it) {
            constexpr int q = decltype(it)::value / TB, j = decltype(it)::value % TB;
            hf[q][j] = lds_read_b128<j * 2048>(at + 2 * W_BYTES + wt * (TB * 2048) + rl_at[q]);
        });
        static_for<2 * MR>([&](auto it) {
            constexpr int q = decltype(it)::value / MR, i = decltype(it)::value % MR;
            bf[q][i] = lds_read_b128<i * 2048>(at + wr * (MR * 2048) + rl_at[q]);
        });
        wait_lgkmcnt<0>();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int i = 0; i < MR; ++i)
#pragma unroll
                for (int j = 0; j < TB; ++j) acc[i][j] = E::mfma16(hf[q][j], bf[q][i], acc[i][j]);
    };

    issue(0, 0);
    if (k_first < blocks) issue_piece(group_of(k_first));
    issue(1, 1);
    int stage = 0;
    auto next = [&](int q) { return q + 1 == STAGES ? 0 : q + 1; };
    // the start of a step: it and its scales have landed, for everyone, and everyone is done with what is refilled now
    auto arrive = [&] {
        __builtin_amdgcn_sched_barrier(0);
        wait_vmcnt<LPS>();                             // (the loads of the step after it)
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };
    for (int step = 0; step < low; ++step) {
        arrive();
        issue(step + 2, next(next(stage)));
        __builtin_amdgcn_sched_barrier(0);
        multiply_low(smem_lds + (uint32_t)stage * STAGE);
        stage = next(stage);
    }
    if (low > 0) {
#pragma unroll
        for (int i = 0; i < MR; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] *= p.s;
    }
    // Beside the products of a round go the reads of the next and its share of the loads two steps ahead: a load takes the CU 16
    // cycles and more, and a wave that issues a step's in one go waits for them (14336 x 4096, 512 tokens: 1300 of 5600 cycles a step).
    constexpr int SHARE = (LPS + ROUNDS - 1) / ROUNDS;
    static_assert(LPS % ROUNDS == 0 || ROUNDS == 4, "loads of a round");
    auto share = [&](auto n_tag, auto blk_tag, int step, int into) {   // the n-th share of a step's loads, spread over the blocks
        constexpr int n = decltype(n_tag)::value, blk = decltype(blk_tag)::value;
        static_for<SHARE>([&](auto l_tag) {
            constexpr int l = decltype(l_tag)::value;
            if constexpr (n * SHARE + l < LPS && blk == l * BLOCKS / SHARE) issue_one(std::integral_constant<int, n * SHARE + l>{}, step, into);
        });
    };
    typedef std::integral_constant<int, 0> H0;
    Round even, odd;
    // the piece that block b begins, if it begins one
    auto issue_next_piece = [&](int b) {
        if (b < k_end && group_of(b) / PIECE != group_of(b - 1) / PIECE) issue_piece(group_of(b));
    };
    auto landed = [] { __builtin_amdgcn_sched_barrier(0); wait_lgkmcnt<0>(); __builtin_amdgcn_sched_barrier(0); };
    if (low < steps) {
        arrive();
        issue_next_piece(k_first + 1);
        static_for<SHARE>([&](auto l) { issue_one(l, low + 2, next(next(stage))); });
        read(H0{}, even, smem_lds + (uint32_t)stage * STAGE, scales_at(k_first));
        landed();                                      // (no read may be on its way at the loop's end: the compiler copies registers there)
    }
    for (int step = low; step < steps; ++step) {
        static_for<ROUNDS>([&](auto h_tag) {
            constexpr int h = decltype(h_tag)::value;
            if constexpr (h + 1 < ROUNDS) {
                const uint32_t at = smem_lds + (uint32_t)stage * STAGE, sat = scales_at(k_first + step - low);
                multiply(h % 2 ? odd : even, [&](auto blk) {
                    __builtin_amdgcn_sched_barrier(0);
                    read_part(std::integral_constant<int, h + 1>{}, blk, h % 2 ? even : odd, at, sat);
                    share(std::integral_constant<int, h + 1>{}, blk, step + 2, next(next(stage)));
                    __builtin_amdgcn_sched_barrier(0);
                });
            } else {                                   // this wave has read all of the step (behind the last one comes a round of zeros)
                arrive();
                const int done = stage, b = k_first + step - low;
                stage = next(stage);
                const uint32_t at = smem_lds + (uint32_t)stage * STAGE, sat = scales_at(b + 1 < k_end ? b + 1 : b);
                issue_next_piece(b + 2);
                multiply(h % 2 ? odd : even, [&](auto blk) {
                    __builtin_amdgcn_sched_barrier(0);
                    read_part(H0{}, blk, even, at, sat);
                    share(H0{}, blk, step + 3, done);
                    __builtin_amdgcn_sched_barrier(0);
                });
            }
            landed();
        });
    }
    wait_vmcnt<0>();                                   // the loads past the end have written their zeros
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    if (whole * BLOCK_K < K && z == p.ksplit - 1) {
        // the columns that the rows end in, a word of codes at a time (a chunk may end past the tensor); zeros past the end
        const uint32_t k0 = (uint32_t)whole * BLOCK_K;
#pragma unroll
        for (int i = 0; i < WL; ++i) {
            const int row = (wave * WL + i) * 16 + (lane >> 2), chunk = (lane & 3) ^ ((row >> 2) & 3);
            u32x4_t v;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                v[q] = __builtin_amdgcn_raw_buffer_load_b32(rw, vw[i] != OUTSIDE && (int)k0 + chunk * 32 + q * 8 < K ? vw[i] + q * 4 : OUTSIDE, k0 / 2, 0);
            lds_write_b128(smem_lds + (uint32_t)((wave * WL + i) * 1024 + lane * 16), make_uint4(v[0], v[1], v[2], v[3]));
        }
#pragma unroll
        for (int i = 0; i < XL; ++i) {
            const int row = (wave * XL + i) * 4 + (lane >> 4), chunk = (lane & 15) ^ (row & 15);
            const u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(rx, (int)k0 + chunk * 8 < K ? vx[i] : OUTSIDE, k0 * 2, 0);
            lds_write_b128(smem_lds + (uint32_t)(W_BYTES + (wave * XL + i) * 1024 + lane * 16), make_uint4(v[0], v[1], v[2], v[3]));
        }
        issue_piece(group_of(whole));
        wait_vmcnt<0>();
        wait_lgkmcnt<0>();
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        static_for<ROUNDS>([&](auto h_tag) {
            if (whole * BLOCK_K + decltype(h_tag)::value * (KS * 32) >= K) return;   // (no scales there either)
            read(h_tag, even, smem_lds, scales_at(whole));
            landed();
            multiply(even, [](auto) {});
        });
        __builtin_amdgcn_s_barrier();
    }

    // lane: tokens 4 lq .. +3 of block j, row l16 of block i.  Through LDS, so that whole vectors along the rows of y are stored.
    float* const red = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int i = 0; i < MR; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                red[(wt * TB * 16 + j * 16 + lq * 4 + e) * RED_LD + wr * MR * 16 + i * 16 + l16] = acc[i][j][e];
    __syncthreads();
    constexpr int EIGHTS = ROWS / 8;
    static_assert(THREADS % EIGHTS == 0, "a thread keeps its columns");
    const int c = (int)threadIdx.x % EIGHTS * 8, n = n0 + c;
    if (c >= rows) return;                             // d_out is a multiple of 8
    float g[8], bias[8];
    if (!p.part || (z == 0 && t0 == 0)) {
        float cj[8], mj[8];
        Eight<float>::load(p.c + n, cj);
        Eight<float>::load(p.m + n, mj);
#pragma unroll
        for (int k = 0; k < 8; ++k) { g[k] = mj[k] / ((cj[k] < p.eps) ? p.eps : cj[k]); bias[k] = 0.f; }
        if (p.part && (int)threadIdx.x < EIGHTS) Eight<float>::store(p.g + n, g);   // for the launch that sums the slices
        if (!p.part && p.bias) Eight16<DT>::load(p.bias + n, bias);
    }
    for (int t = (int)threadIdx.x / EIGHTS; t < toks; t += THREADS / EIGHTS) {
        float v[8];
        Eight<float>::load(red + t * RED_LD + c, v);
        if (p.part) { Eight<float>::store(p.part + ((int64_t)z * T + t0 + t) * N + n, v); continue; }
        const int64_t at = (int64_t)(t0 + t) * N + n;
        if (p.inner) Eight16<DT>::store(p.inner + at, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = fmaf(g[k], v[k], bias[k]);
        Eight16<DT>::store(p.y + at, v);
    }
}

constexpr int SMALL_TOK = 64, SMALL_ROWS = 128, LARGE_TOK = 128, LARGE_ROWS = 256;

// The tile and the slices of the columns that are the cheapest, in tenths of a microsecond: a step of a small tile 12 while every
// workgroup has a CU to itself and 17 where two share one, of a large tile 24 (four times the products), 60 for what comes before the
// first step and behind the last; and where there are slices 40 for the launch that sums them, and the partial sums written and read at
// 4 TB/s.  At most eight slices of four steps at least.  Groups of 32: small tiles (the large one's scales and codes do not fit the
// registers).  (Forward, h in slices in both, us, small / large: 4096 x 4096, r 64, 128 tokens 40.0 / 49.4; 14336 x 4096, 128 tokens
// 60.3 / 56.1; 8192 x 8192, 256 tokens 88.9 / 77.7; 27648 x 5120, 256 tokens 158 / 112.)
struct Choice { bool small; int slices; };
Choice choose(int64_t tokens, int64_t d_out, int64_t d_in, int group_shift)
{
    Choice best{true, 1};
    int64_t least = -1;
    for (int k = 0; k < (group_shift < 6 ? 1 : 2); ++k) {
        const bool small = k == 0;
        const int64_t rows = small ? SMALL_ROWS : LARGE_ROWS, tok = small ? SMALL_TOK : LARGE_TOK;
        const int64_t tiles = (d_out + rows - 1) / rows * ((tokens + tok - 1) / tok), steps = (d_in + BLOCK_K - 1) / BLOCK_K;
        for (int64_t ks = 1; ks <= 8 && (ks == 1 || steps >= 4 * ks); ++ks) {
            const int64_t wgs = tiles * ks, at_once = small ? 512 : 256, step = small ? (wgs <= 256 ? 12 : 17) : 24;
            const int64_t cost = (wgs + at_once - 1) / at_once * ((steps + ks - 1) / ks * step + 60) + (ks > 1 ? 40 + ks * tokens * d_out / 50000 : 0);
            if (least < 0 || cost < least) { least = cost; best = Choice{small, (int)ks}; }
        }
    }
    return best;
}

template <int CODE, int SUB, bool ZERO, int DT>
hipError_t launch_shape(const QuantTileArgs& a, hipStream_t st)
{
    const dim3 grid((unsigned)((int64_t)a.row_tiles * a.token_tiles * a.ksplit));
    if constexpr (SUB > 1)
        if (!choose(a.T, a.w.d_out, a.w.d_in, a.w.group_shift).small) {
            quant_tile_kernel<4, 2, 4, 4, CODE, SUB, ZERO, DT><<<grid, dim3(512), 0, st>>>(a);
            return hipGetLastError();
        }
    quant_tile_kernel<4, 1, 2, 4, CODE, SUB, ZERO, DT><<<grid, dim3(256), 0, st>>>(a);
    return hipGetLastError();
}
template <int SUB, int DT>
hipError_t launch_code(const QuantTileArgs& a, hipStream_t st)
{
    if (a.w.code == DORA_QUANT_FP4) return launch_shape<DORA_QUANT_FP4, SUB, false, DT>(a, st);
    return a.w.zero ? launch_shape<DORA_QUANT_INT4, SUB, true, DT>(a, st) : launch_shape<DORA_QUANT_INT4, SUB, false, DT>(a, st);
}
template <int DT>
hipError_t launch(const QuantTileArgs& a, hipStream_t st)
{
    if (a.w.group_shift >= 7) return launch_code<4, DT>(a, st);
    return a.w.group_shift == 6 ? launch_code<2, DT>(a, st) : launch_code<1, DT>(a, st);
}

}  // namespace

int quant_tile_slices(int64_t tokens, const QuantWeight& w) { return choose(tokens, w.d_out, w.d_in, w.group_shift).slices; }

hipError_t launch_quant_tile(QuantTileArgs a, int dt, hipStream_t st)
{
    TraceScope ts(DORA_K_QUANT_TILE, st);
    const bool small = choose(a.T, a.w.d_out, a.w.d_in, a.w.group_shift).small;
    a.token_tiles = (a.T + (small ? SMALL_TOK : LARGE_TOK) - 1) / (small ? SMALL_TOK : LARGE_TOK);
    a.row_tiles = (a.w.d_out + (small ? SMALL_ROWS : LARGE_ROWS) - 1) / (small ? SMALL_ROWS : LARGE_ROWS);
    return dt == DT_F16 ? launch<DT_F16>(a, st) : launch<DT_BF16>(a, st);
}

}  // namespace dora
