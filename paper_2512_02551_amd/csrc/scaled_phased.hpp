// The product of 8-bit floats for large tiles: a block of K in four phases.
//
// What bounds it: the matrix cores, as long as the copies of the next blocks land in time.  Two buffers of a 256 x 256 tile fill the
// LDS, so a buffer cannot wait until all of it has been read: a block of K is four units -- the upper and lower half of the A tile, two
// halves of the B tile -- and a unit is refilled as soon as its fragments are in registers.  F is the half of B that a block begins with (the left
// one in even blocks, the right one in odd ones), S the other:
//
//   phase  multiplies  reads (LDS -> registers)                     copies (memory -> LDS)
//   1      A0 x F      S of this block                              A1 of the next block, first half
//   2      A0 x S      A1, each fragment in place of A0's           A1 of the next block, second half
//   3      A1 x S                                                   A0, F, scales of the block after the next
//   4      A1 x F      F and A0 of the next block, in place         S of the block after the next
//
// Every fragment has one place in registers for half of a block: 128 sums, 64 registers of fragments and 16 for sums on their way to the scales
// leave the rest of 256 for addresses.  Two barriers a block, in front of phases 1 and 3: a unit is refilled behind the barrier that follows the
// last instruction that needed its fragments, so no wave has to wait for its LDS reads there; and copies are waited for a whole block
// (four phases) after they were issued, so what is still in flight at a barrier is a compile-time constant.
//
// Measured back to back on several cards, bf16 C: 4001 x 14336 x 4096, f32 scales 208 .. 222 us (2.1 .. 2.2 PFLOP/s; the matrix cores busy half of the cycles at
// 1.9 GHz), 11008 x 4096 x 8064, e8m0 scales 264 .. 280 us (2.6 .. 2.8 PFLOP/s); 4001 x 4 rows of 32 experts, 4096 x 4096, 298 .. 314 us (1.7 .. 1.8 PFLOP/s of
// rows that exist; with e8m0 scales 270).  fp32 C, 128 x 128: 16 experts' 4096 x 2048 over 8192 rows 194 .. 207 us (0.7 PFLOP/s, 2.7 TB/s of stores).
// What is left with f32 scales: the multiply-adds for the scales, 128 a lane and block, are issued beside the matrix instructions (1.6 us a block, 1.3 in a library product with one scale), and a tile's start and end, 8
// us, which nothing covers as one workgroup fills the LDS.
#pragma once
#include "scaled_tile.hpp"

// The loop is in the kernel twice; not inlined, its lambdas would put the fragments in memory.
#define HGEMM_INLINED __attribute__((always_inline))

namespace hgemm {

template <int BM_, int BN_, int WAVES_M_, int WAVES_N_> struct ScaledPhasedCfg {
    static constexpr int BM = BM_, BN = BN_, WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, STAGES = 0;
    static constexpr int NWAVES = WAVES_M * WAVES_N, THREADS = 64 * NWAVES;
    static constexpr int HM = BM / 2, HN = BN / 2, QM = HM / WAVES_M, QN = HN / WAVES_N, TM = QM / 16, TN = QN / 16;
    static constexpr int A_UNIT = HM * 128, B_UNIT = HN * 128, B_BASE = 4 * A_UNIT;         // A units (buffer, half), then B units
    static constexpr int AL = HM / 8 / NWAVES, BL = HN / 8 / NWAVES;                        // copies per wave and unit
    static constexpr int SLOADS = (BM + BN) / 64 / NWAVES, SCALE_BYTES = (BM + BN) * 4, SCALE_BASE = 4 * (A_UNIT + B_UNIT), SCALE_BUFFERS = 4;
    static constexpr int GROUP = AL + 2 * BL + SLOADS;                                      // copies of phase 3
    static constexpr int LOOP_BYTES = SCALE_BASE + SCALE_BUFFERS * SCALE_BYTES;
    static constexpr int OUT_BYTES = BM * (BN * (4 * TM * TN <= 16 ? 4 : 2) + 16), LDS_BYTES = LOOP_BYTES > OUT_BYTES ? LOOP_BYTES : OUT_BYTES;
    static_assert(QM % 16 == 0 && QN % 16 == 0 && 128 % QN == 0, "a wave's share of a quadrant");
    static_assert(HM % (8 * NWAVES) == 0 && HN % (8 * NWAVES) == 0 && (BM + BN) % (64 * NWAVES) == 0 && BM % 64 == 0, "units split into wave loads");
    static_assert(NWAVES % 2 == 0, "one swizzle serves all of a lane's copies");
    static_assert(HN % 128 == 0 || 128 % HN == 0, "scales of B");
    static_assert(LDS_BYTES <= 160 * 1024, "LDS");
};

template <class C, int SUM, bool A5, bool B_BY_ROW>
__global__ __launch_bounds__(C::THREADS, C::LDS_BYTES > 80 * 1024 || C::NWAVES >= 8 ? 1 : 2) void scaled_phased_kernel(ScaledArgs a)
{
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    constexpr bool WIDE = SUM == SUM_WIDE || SUM == SUM_WIDE_E8M0, byte = SUM == SUM_E8M0 || SUM == SUM_WIDE_E8M0;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, lg = lane >> 4;
    const int wm = wave / C::WAVES_N * C::QM, wn = wave % C::WAVES_N * C::QN;
    unsigned mt, nt;
    tile_coords(blockIdx.x, a, mt, nt);
    ScaledTile tile;
    if (!find_tile(a, (int)mt, C::BM, tile)) return;
    const int n0 = (int)nt * C::BN;

    f4 acc[2][2][C::TM][C::TN];
#pragma unroll
    for (int i = 0; i < 4 * C::TM * C::TN; ++i) (&acc[0][0][0][0])[i] = f4{0.f, 0.f, 0.f, 0.f};

    const int kb0 = tile.k_begin / kScaleBlock, blocks = tile.zero ? 0 : (tile.k_end + kScaleBlock - 1) / kScaleBlock - kb0;
    if (blocks > 0) {
        const unsigned OOB = 0x80000000u;
        const uint8_t* base_a = (a.a_rows ? a.A : a.A + (int64_t)tile.m0 * a.lda) + tile.k_begin;
        const uint8_t* base_b = a.B + (b_group(a, tile) + n0) * a.ldb + tile.k_begin;
        const int k_len = tile.k_end - tile.k_begin;
        const int4v rsrcA = make_rsrc(base_a, (unsigned)(a.a_rows ? a.a_rows : min(C::BM, tile.m_end - tile.m0)) * (unsigned)a.lda - tile.k_begin);
        const int4v rsrcB = make_rsrc(base_b, (unsigned)min(C::BN, a.N - n0) * (unsigned)a.ldb - tile.k_begin);
        // wave-load j of a unit covers its rows 8 (j NWAVES + wave) ..; lane i fills place i % 8 of row i / 8
        const int chunk = (lane & 7) ^ (4 * (wave & 1) + (lane >> 4));
        unsigned va[2][C::AL], vb[2][C::BL];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < C::AL; ++j) {
                const int row = h * C::HM + (j * C::NWAVES + wave) * 8 + (lane >> 3);
                const int r = row_of_a(a, tile.m0 + row, tile.m_end);
                va[h][j] = r < 0 ? OOB : (unsigned)(a.a_rows ? r : row) * (unsigned)a.lda + chunk * 16;
            }
#pragma unroll
            for (int j = 0; j < C::BL; ++j) {
                const int row = h * C::HN + (j * C::NWAVES + wave) * 8 + (lane >> 3);
                vb[h][j] = n0 + row >= a.N ? OOB : (unsigned)row * (unsigned)a.ldb + chunk * 16;
            }
        }
        const int ssize = byte ? 1 : 4;
        const char* base_sa = (const char*)a.SA + ((a.a_rows ? 0 : tile.m0) + kb0 * a.ldsa) * ssize;
        const char* base_sb = (const char*)a.SB + (B_BY_ROW ? n0 + kb0 * a.ldsb : sb_group(a, tile) + (int64_t)(n0 / kScaleBlock) * a.ldsb + kb0) * ssize;
        const int64_t step_sa = a.ldsa * ssize, step_sb = (B_BY_ROW ? a.ldsb : 1) * ssize;
        unsigned vs[C::SLOADS];
#pragma unroll
        for (int j = 0; j < C::SLOADS; ++j) {
            const int row = (j * C::NWAVES + wave) * 64 + lane, r = row - C::BM;
            if (row < C::BM) {
                const int ra = row_of_a(a, tile.m0 + row, tile.m_end);
                vs[j] = ra < 0 ? OOB : (unsigned)(a.a_rows ? ra : row) * ssize;
            } else {
                vs[j] = n0 + r >= a.N ? OOB : (unsigned)(B_BY_ROW ? r : (int64_t)(r / kScaleBlock) * a.ldsb) * ssize;
            }
        }
        const unsigned lds0 = __builtin_amdgcn_readfirstlane((int)lds_addr_of(lds));
        // copies of block t; chunks past K and blocks past the last are zeros
        auto copy_a = [&](int t, auto buf, auto h, auto j) HGEMM_INLINED {
            constexpr int at = (decltype(buf)::value * 2 + decltype(h)::value) * C::A_UNIT + decltype(j)::value * C::NWAVES * 1024;
            copy16(rsrcA, lds0 + at + wave * 1024, t * kScaleBlock + chunk * 16 < k_len ? va[h][j] : OOB, (unsigned)t * kScaleBlock);
        };
        auto copy_b = [&](int t, auto buf, auto h, auto j) HGEMM_INLINED {
            constexpr int at = C::B_BASE + (decltype(buf)::value * 2 + decltype(h)::value) * C::B_UNIT + decltype(j)::value * C::NWAVES * 1024;
            copy16(rsrcB, lds0 + at + wave * 1024, t * kScaleBlock + chunk * 16 < k_len ? vb[h][j] : OOB, (unsigned)t * kScaleBlock);
        };
        auto copy_s = [&](int t, auto j) HGEMM_INLINED {
            const int first = (decltype(j)::value * C::NWAVES + wave) * 64;
            const int4v r = make_rsrc(first < C::BM ? base_sa : base_sb, t < blocks ? 0x7fffffffu : 0u);
            copy_scale<byte>(r, lds0 + C::SCALE_BASE + (t & (C::SCALE_BUFFERS - 1)) * C::SCALE_BYTES + first * 4, vs[j]);
            if constexpr (decltype(j)::value == C::SLOADS - 1) {
                base_sa += step_sa;
                base_sb += step_sb;
            }
        };
        // copy x of phase 3's group for block t, whose first half of B is `f`: A0, F, scales, S
        auto copy_group = [&](int t, auto buf, auto f, auto x_tag) HGEMM_INLINED {
            constexpr int x = decltype(x_tag)::value;
            if constexpr (x < C::AL) copy_a(t, buf, ic<0>{}, ic<x>{});
            else if constexpr (x < C::AL + C::BL) copy_b(t, buf, f, ic<x - C::AL>{});
            else if constexpr (x < C::AL + C::BL + C::SLOADS) copy_s(t, ic<x - C::AL - C::BL>{});
            else copy_b(t, buf, ic<1 - decltype(f)::value>{}, ic<x - C::AL - C::BL - C::SLOADS>{});
        };

        // fragments: chunks lg and lg + 4 of a row
        const int ra = wm + l16, rb = wn + l16;
        const int at_a = ra * 128 + ((lg ^ ((ra >> 1) & 7)) << 4), at_b = C::B_BASE + rb * 128 + ((lg ^ ((rb >> 1) & 7)) << 4);
        const int at_sa = C::SCALE_BASE + ra * 4, at_sb = C::SCALE_BASE + (C::BM + (SUM == SUM_E8M0 ? rb : wn + 4 * lg)) * 4;
        Fragment<WIDE> fa[C::TM], fb[2][C::TN];
        Chunks ra_new[WIDE ? C::TM : 1], rb_new[WIDE ? C::TN : 1];     // WIDE: read, not yet turned into fp16
        int ia[C::TM], ib[2][C::TN];                    // scales as they lie
        i4 sb[2][C::TN];
        auto value = [&](int raw) HGEMM_INLINED { return byte ? e8m0_value(raw) : __builtin_bit_cast(float, raw); };
        auto read_a = [&](int t, auto buf, auto h, auto tm_tag) HGEMM_INLINED {
            constexpr int tm = decltype(tm_tag)::value, at = (decltype(buf)::value * 2 + decltype(h)::value) * C::A_UNIT + tm * 2048;
            if constexpr (WIDE) ra_new[tm].read(lds + at_a + at, lds + (at_a ^ 64) + at);
            else fa[tm] = make_fragment<WIDE, A5>(*(const i4*)(lds + at_a + at), *(const i4*)(lds + (at_a ^ 64) + at));
            ia[tm] = *(const int*)(lds + at_sa + (t & (C::SCALE_BUFFERS - 1)) * C::SCALE_BYTES + (decltype(h)::value * C::HM + tm * 16) * 4);
        };
        auto read_b = [&](int t, auto buf, auto q, auto tn_tag) HGEMM_INLINED {
            constexpr int tn = decltype(tn_tag)::value, Q = decltype(q)::value, at = (decltype(buf)::value * 2 + Q) * C::B_UNIT + tn * 2048;
            if constexpr (WIDE) rb_new[tn].read(lds + at_b + at, lds + (at_b ^ 64) + at);
            else fb[Q][tn] = make_fragment<WIDE, false>(*(const i4*)(lds + at_b + at), *(const i4*)(lds + (at_b ^ 64) + at));
            const char* s = lds + at_sb + (t & (C::SCALE_BUFFERS - 1)) * C::SCALE_BYTES + (Q * C::HN + tn * 16) * 4;
            if constexpr (SUM == SUM_E8M0) {
                ib[Q][tn] = *(const int*)s;
            } else if constexpr (B_BY_ROW) {
                sb[Q][tn] = *(const i4*)s;
            } else if constexpr (tn == 0) {
                ib[Q][0] = *(const int*)s;              // one scale for all of a wave's columns of a half
            }
        };

        // The sums of a tile wait DELAY tiles for their multiply-adds (across phases), so that those run under later matrix instructions.  A tile of
        // the same column then waits no longer than the scales of that column stay in place.
        constexpr int TILES = C::TM * C::TN, DELAY = C::TN;
        f4 p[WIDE ? 2 * C::TN : DELAY];                 // WIDE: of two rows of tiles in turn
        float scale_of[DELAY];
        auto add = [&](auto h, auto q, auto i_tag) HGEMM_INLINED {
            constexpr int i = decltype(i_tag)::value, tm = i / C::TN, tn = i % C::TN;
            f4& to = acc[decltype(h)::value][decltype(q)::value][tm][tn];
#pragma unroll
            for (int e = 0; e < 4; ++e) to[e] += p[i % DELAY][e] * (B_BY_ROW ? scale_of[i % DELAY] * value(sb[decltype(q)::value][tn][e]) : scale_of[i % DELAY]);
            asm volatile("" : "+v"(to));                // here, not behind later matrix instructions
        };
        // WIDE: a row of tiles, whose fp16 instructions go tile by tile in turn (those of one tile wait for each other), then the multiply-adds of the row
        // before.
        auto add_row = [&](auto h, auto q, auto tm_tag) HGEMM_INLINED {
            constexpr int tm = decltype(tm_tag)::value, H = decltype(h)::value, Q = decltype(q)::value;
            static_for<C::TN>([&](auto tn) HGEMM_INLINED {
                f4& to = acc[H][Q][tm][tn];
                const f4 x = p[(tm & 1) * C::TN + tn];
#pragma unroll
                for (int e = 0; e < 4; ++e) to[e] += x[e] * (B_BY_ROW ? scale_of[tm & 1] * value(sb[Q][tn][e]) : scale_of[tm & 1]);
                asm volatile("" : "+v"(to));
            });
        };
        static_assert(!WIDE || (C::TM % 2 == 0 && C::TN >= 2), "rows of tiles take turns");
        auto phase_wide = [&](auto h, auto q, auto ph, auto pq, auto first, auto new_a, auto new_b, auto&& side) HGEMM_INLINED {
            constexpr int Q = decltype(q)::value;
            static_for<C::TM>([&](auto tm_tag) HGEMM_INLINED {
                constexpr int tm = decltype(tm_tag)::value;
                if constexpr (decltype(new_a)::value) fa[tm] = make_fragment<WIDE, A5>(ra_new[tm].lo, ra_new[tm].hi);
                if constexpr (decltype(new_b)::value && tm == 0)
                    static_for<C::TN>([&](auto tn) HGEMM_INLINED { fb[Q][tn] = make_fragment<WIDE, false>(rb_new[tn].lo, rb_new[tn].hi); });
                static_for<4>([&](auto k) HGEMM_INLINED {
                    static_for<C::TN>([&](auto tn) HGEMM_INLINED {
                        f4& x = p[(tm & 1) * C::TN + tn];
                        x = __builtin_amdgcn_mfma_f32_16x16x32_f16(fb[Q][tn].v[k], fa[tm].v[k], k ? x : f4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
                    });
                });
                if constexpr (tm > 0) add_row(h, q, ic<tm - 1>{});
                else if constexpr (!decltype(first)::value) add_row(ph, pq, ic<C::TM - 1>{});
                scale_of[tm & 1] = B_BY_ROW ? value(ia[tm]) : value(ia[tm]) * value(ib[Q][0]);
                static_for<C::TN>([&](auto tn) HGEMM_INLINED { side(ic<tm * C::TN + decltype(tn)::value>{}); });
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        // Quadrant (h, q), after quadrant (ph, pq); side(i) is what follows instruction i.  new_a, new_b: the fragments are used for the first time.
        auto phase = [&](auto h, auto q, auto ph, auto pq, auto first, auto new_a, auto new_b, auto&& side) HGEMM_INLINED {
            if constexpr (WIDE) {
                phase_wide(h, q, ph, pq, first, new_a, new_b, side);
                return;
            }
            constexpr int H = decltype(h)::value, Q = decltype(q)::value;
            static_for<TILES>([&](auto i_tag) HGEMM_INLINED {
                constexpr int i = decltype(i_tag)::value, tm = i / C::TN, tn = i % C::TN;
                if constexpr (SUM == SUM_E8M0) {
                    acc[H][Q][tm][tn] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[Q][tn].v, fa[tm].v, acc[H][Q][tm][tn], 0, A5 ? 1 : 0, 0, ib[Q][tn], 0, ia[tm]);
                    if constexpr (C::NWAVES >= 8) asm volatile("" : "+v"(acc[H][Q][tm][tn]));
                } else {
                    if constexpr (i >= DELAY) add(h, q, ic<i - DELAY>{});
                    else if constexpr (!decltype(first)::value) add(ph, pq, ic<TILES - DELAY + i>{});
                    p[i % DELAY] = mma_block<A5>(fb[Q][tn], fa[tm], f4{0.f, 0.f, 0.f, 0.f});
                    scale_of[i % DELAY] = B_BY_ROW ? value(ia[tm]) : value(ia[tm]) * value(ib[Q][0]);
                }
                side(i_tag);
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        static_assert(TILES % DELAY == 0, "the places of waiting sums go round with the tiles");
        // The multiply-adds that still wait, of quadrant (h, q); what the next phase then finds waiting is zeros.
        auto settle = [&](auto h, auto q) HGEMM_INLINED {
            if constexpr (SUM == SUM_E8M0) return;
            if constexpr (WIDE) add_row(h, q, ic<C::TM - 1>{});
            else static_for<DELAY>([&](auto x) HGEMM_INLINED { add(h, q, ic<TILES - DELAY + decltype(x)::value>{}); });
            static_for<sizeof p / sizeof p[0]>([&](auto x) HGEMM_INLINED { p[x] = f4{0.f, 0.f, 0.f, 0.f}; });
            static_for<DELAY>([&](auto x) HGEMM_INLINED { scale_of[x] = 0.f; });
        };
        auto block = [&](int t, auto parity, auto first, auto half) HGEMM_INLINED {
            constexpr bool HALF = decltype(half)::value;
            typedef ic<decltype(parity)::value> P;
            typedef ic<1 - decltype(parity)::value> R;  // the other buffer, the second half of B
            typedef ic<0> Z;
            typedef ic<1> O;
            // copies go out evenly: a burst fills the queue to memory, and a wave that waits for its place there issues no matrix instruction either
            auto side12 = [&](auto i) HGEMM_INLINED {
                constexpr int s = decltype(i)::value, lo = s * C::AL / (2 * TILES), hi = (s + 1) * C::AL / (2 * TILES);
                static_for<hi - lo>([&](auto x) HGEMM_INLINED { copy_a(t + 1, R{}, O{}, ic<lo + decltype(x)::value>{}); });     // HALF: zeros, which keeps the count
            };
            wait_vmcnt<C::GROUP>();
            asm volatile("s_barrier" ::: "memory");
            phase(Z{}, P{}, O{}, R{}, first, O{}, O{}, [&](auto i) HGEMM_INLINED {       // the block before ended with A1 and its own F, which is this one's S
                side12(ic<i>{});
                if constexpr (i < C::TN) read_b(t, P{}, R{}, i);
            });
            phase(Z{}, R{}, Z{}, P{}, Z{}, Z{}, O{}, [&](auto i) HGEMM_INLINED {
                side12(ic<TILES + i>{});
                if constexpr (i % C::TN == C::TN - 1)
                    if constexpr (!HALF) read_a(t, P{}, O{}, ic<i / C::TN>{});
            });
            wait_vmcnt<C::AL + C::BL>();
            asm volatile("s_barrier" ::: "memory");
            auto copies = [&](auto i) HGEMM_INLINED {
                constexpr int s = decltype(i)::value, lo = s * C::GROUP / (2 * TILES), hi = (s + 1) * C::GROUP / (2 * TILES);
                static_for<hi - lo>([&](auto x) HGEMM_INLINED { copy_group(t + 2, P{}, P{}, ic<lo + decltype(x)::value>{}); });
            };
            auto side3 = [&](auto i) HGEMM_INLINED { copies(i); };
            auto side4 = [&](auto i) HGEMM_INLINED {
                copies(ic<TILES + i>{});
                if constexpr (i < C::TN) read_b(t + 1, R{}, R{}, i);
                if constexpr (i % C::TN == C::TN - 1) read_a(t + 1, R{}, Z{}, ic<i / C::TN>{});
            };
            if constexpr (!HALF) {
                phase(O{}, R{}, Z{}, R{}, Z{}, O{}, Z{}, side3);
                phase(O{}, P{}, O{}, R{}, Z{}, Z{}, Z{}, side4);
            } else {
                settle(Z{}, R{});
                static_for<TILES>(side3);
                static_for<TILES>(side4);
            }
        };

        // A tile of no more than half the rows has no A1: its phases 3 and 4 only move data.  Groups of rows end in such tiles every other time.  (A loop
        // of its own: a branch inside one loop costs hundreds of registers.)
        auto all_blocks = [&](auto half) HGEMM_INLINED {
            // the first two blocks, as the phases would have copied them
            static_for<C::GROUP>([&](auto x) HGEMM_INLINED { copy_group(0, ic<0>{}, ic<0>{}, x); });
            static_for<C::AL>([&](auto j) HGEMM_INLINED { copy_a(0, ic<0>{}, ic<1>{}, j); });
            static_for<C::GROUP>([&](auto x) HGEMM_INLINED { copy_group(1, ic<1>{}, ic<1>{}, x); });
            wait_vmcnt<C::GROUP>();
            asm volatile("s_barrier" ::: "memory");
            static_for<C::TN>([&](auto tn) HGEMM_INLINED { read_b(0, ic<0>{}, ic<0>{}, tn); });
            static_for<C::TM>([&](auto tm) HGEMM_INLINED { read_a(0, ic<0>{}, ic<0>{}, tm); });
            block(0, ic<0>{}, ic<1>{}, half);
            int t = 1;
#pragma unroll 1
            for (; t + 1 < blocks; t += 2) {
                block(t, ic<1>{}, ic<0>{}, half);
                block(t + 1, ic<0>{}, ic<0>{}, half);
            }
            // sums that still wait: of the last quadrant, A1 x F
            if (t < blocks) {
                block(t, ic<1>{}, ic<0>{}, half);
                if constexpr (!decltype(half)::value) settle(ic<1>{}, ic<1>{});
            } else {
                if constexpr (!decltype(half)::value) settle(ic<1>{}, ic<0>{});
            }
        };
        if (tile.m_end - tile.m0 > C::HM) all_blocks(ic<0>{});
        else all_blocks(ic<1>{});
        wait_vmcnt<0>();
    }
    __syncthreads();
    store_tile<C, WIDE>(lds, a, tile, n0, [&](auto&& put) {
        static_for<2>([&](auto h) { static_for<2>([&](auto q) {
#pragma unroll
            for (int i = 0; i < C::TM; ++i)
#pragma unroll
                for (int j = 0; j < C::TN; ++j) put(h * C::HM + wm + i * 16 + l16, q * C::HN + wn + j * 16 + 4 * lg, acc[h][q][i][j]);
        }); });
    });
}

}  // namespace hgemm
