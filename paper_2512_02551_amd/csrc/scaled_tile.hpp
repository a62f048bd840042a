// The product of 8-bit floats: tiles of A and B through LDS (copies straight from memory, STAGES blocks of K deep).
//
// A stage is one block of K of the tile's rows, 128 bytes a row in a swizzle of 16-byte chunks that keeps both the copies and the fragments' reads free of
// conflicts, and the block's scales.  What bounds it: small tiles wait for memory -- 16 x 64 ones stream the weights of experts with a few
// rows each, 24 x 4 rows of 32 experts of 4096 x 2048 in 42 us (219 MB of weights that have rows: 5.2 TB/s; four stages leave room for three workgroups a
// unit, which cover each other's starts: six stages and two 46 us, three and four 43, but 78 for 72 on 8 x 2 of 8 of 14336 x 4096) -- large ones for
// the LDS and the multiply-adds of the scales, one for each sum and block: 256 x 256 tiles take 257 us of 4001 x 14336 x 4096, phased ones 208 .. 222.  They serve the
// K and tile shapes that those do not.
#pragma once
#include "scaled_product.hpp"

namespace hgemm {

// How a block of K becomes part of the sums.
//   SUM_SCALED  8-bit instructions from zero, one multiply-add with sa * sb for each sum
//   SUM_E8M0    8-bit instructions that apply both scales and add to the sums themselves
//   SUM_WIDE    as SUM_SCALED, on fp16 instructions (C in fp32); SUM_WIDE_E8M0: with scales of a byte
enum { SUM_SCALED = 0, SUM_E8M0 = 1, SUM_WIDE = 2, SUM_WIDE_E8M0 = 3, SUM_KINDS = 4 };

template <int BM_, int BN_, int WAVES_M_, int WAVES_N_, int STAGES_> struct ScaledCfg {
    static constexpr int BM = BM_, BN = BN_, WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, STAGES = STAGES_;
    static constexpr int NWAVES = WAVES_M * WAVES_N, THREADS = 64 * NWAVES;
    static constexpr int WTM = BM / WAVES_M, WTN = BN / WAVES_N, TM = WTM / 16, TN = WTN / 16;
    static constexpr int ROW_LOADS = (BM + BN) / 8, LOADS = (ROW_LOADS + NWAVES - 1) / NWAVES;           // copies of 8 rows; of them, per wave
    static constexpr int SA_LOADS = (BM + 63) / 64, SB_LOADS = (BN + 63) / 64, SLOADS = (SA_LOADS + SB_LOADS + NWAVES - 1) / NWAVES;   // copies of 64 scales
    static constexpr int ALL_LOADS = LOADS + SLOADS;
    static constexpr int ROWS_BYTES = LOADS * NWAVES * 1024, SCALE_BYTES = SLOADS * NWAVES * 256;
    static constexpr int STAGE_BYTES = ROWS_BYTES + SCALE_BYTES, LOOP_BYTES = STAGES * STAGE_BYTES;
    static constexpr int OUT_BYTES = BM * (BN * (TM * TN <= 16 ? 4 : 2) + 16), LDS_BYTES = LOOP_BYTES > OUT_BYTES ? LOOP_BYTES : OUT_BYTES;     // fp32 tiles: store_tile
    static_assert(WTM % 16 == 0 && WTN % 16 == 0 && BM % 16 == 0 && BN % 16 == 0, "wave tile");
    static_assert(NWAVES % 2 == 0, "one swizzle serves all of a lane's copies");
    static_assert(WTN <= 128 && 128 % WTN == 0, "the columns of a wave share a scale of B");
    static_assert(LDS_BYTES <= 160 * 1024, "LDS");
    static_assert(ALL_LOADS * (STAGES - 1) <= 63, "vmcnt is 6 bits");
};

// As dma16, with a wave-uniform offset on top, and for one scale a lane (a byte is widened to four).
__device__ __forceinline__ void copy16(int4v rsrc, unsigned lds_addr, unsigned voff, unsigned soff)
{
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" : : "v"(voff), "s"(rsrc), "s"(soff), "{m0}"(__builtin_amdgcn_readfirstlane((int)lds_addr)) : "memory");
}
template <bool BYTE> __device__ __forceinline__ void copy_scale(int4v rsrc, unsigned lds_addr, unsigned voff)
{
    if constexpr (BYTE) asm volatile("s_nop 0\n\tbuffer_load_ubyte %0, %1, 0 offen lds" : : "v"(voff), "s"(rsrc), "{m0}"(__builtin_amdgcn_readfirstlane((int)lds_addr)) : "memory");
    else asm volatile("s_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" : : "v"(voff), "s"(rsrc), "{m0}"(__builtin_amdgcn_readfirstlane((int)lds_addr)) : "memory");
}

// The tile's sums to C, through LDS: each(put) calls put(row, column, four sums) for all of the calling lane's, then whole rows go out in 16-byte
// stores.  (Eight-byte stores from registers, 32 bytes of a row at a time, cost 50 of 250 us on 4096 x 16384 x 4096.)  The stores bypass
// what they can of the caches: all workgroups of a round end together, and 16 experts' 4096 x 2048 gradients in fp32 take 197 us with it, 234 without.  The
// caller sees to it that nobody uses the LDS any more.
template <class C, class T, class Each> __device__ __forceinline__ void store_tile_as(char* lds, const ScaledArgs& a, const ScaledTile& tile, int n0, Each&& each)
{
    constexpr int PITCH = C::BN * sizeof(T) + 16, PER = 16 / sizeof(T), CPR = C::BN / PER;
    each([&](int row, int col, f4 v) { *(typename Packed4<T>::type*)(lds + row * PITCH + col * sizeof(T)) = pack4<T>(v); });
    __syncthreads();
    T* const first = c_row<T>(a, tile, tile.m0) + n0;
    const int rows = tile.m_end - tile.m0, cols = a.N - n0;
    const bool wide = (((uintptr_t)a.C | (uintptr_t)(a.ldc * sizeof(T))) & 15) == 0 && a.N % PER == 0;
    if (wide) {
#pragma unroll 4
        for (int i = threadIdx.x; i < C::BM * CPR; i += C::THREADS) {
            const int r = i / CPR, n = i % CPR * PER;
            if (r < rows && n < cols) __builtin_nontemporal_store(*(const u4*)(lds + r * PITCH + n * sizeof(T)), (u4*)(first + r * a.ldc + n));
        }
        return;
    }
#pragma unroll 4
    for (int i = threadIdx.x; i < C::BM * C::BN / 4; i += C::THREADS) {
        const int r = i / (C::BN / 4), n = i % (C::BN / 4) * 4;
        if (r >= rows || n >= cols) continue;
        typename Packed4<T>::type v = *(const typename Packed4<T>::type*)(lds + r * PITCH + n * sizeof(T));
        T* const p = first + r * a.ldc + n;
        if (cols - n >= 4) {
            __builtin_memcpy(p, &v, sizeof v);
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (n + e < cols) p[e] = v[e];
        }
    }
}
template <class C, bool WIDE, class Each> __device__ __forceinline__ void store_tile(char* lds, const ScaledArgs& a, const ScaledTile& tile, int n0, Each&& each)
{
    if constexpr (WIDE) store_tile_as<C, float>(lds, a, tile, n0, each);
    else if (a.c_type == HGEMM_F16) store_tile_as<C, _Float16>(lds, a, tile, n0, each);
    else store_tile_as<C, __bf16>(lds, a, tile, n0, each);
}

template <class C, int SUM, bool A5, bool B_BY_ROW>
__global__ __launch_bounds__(C::THREADS, C::LDS_BYTES > 80 * 1024 || C::NWAVES >= 8 ? 1 : 2) void scaled_tile_kernel(ScaledArgs a)
{
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    constexpr bool WIDE = SUM == SUM_WIDE || SUM == SUM_WIDE_E8M0, byte = SUM == SUM_E8M0 || SUM == SUM_WIDE_E8M0;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, lg = lane >> 4;
    const int wm = wave / C::WAVES_N * C::WTM, wn = wave % C::WAVES_N * C::WTN;
    unsigned mt, nt;
    tile_coords(blockIdx.x, a, mt, nt);
    ScaledTile tile;
    if (!find_tile(a, (int)mt, C::BM, tile)) return;
    const int n0 = (int)nt * C::BN;

    f4 acc[C::TM][C::TN];
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int j = 0; j < C::TN; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};

    const int kb0 = tile.k_begin / kScaleBlock, kb1 = tile.zero ? kb0 : (tile.k_end + kScaleBlock - 1) / kScaleBlock;
    const unsigned OOB = 0x80000000u;
    // A row and B row of this lane's copies: copy i of a block covers LDS rows 8 i .. 8 i + 7, A's rows first
    const uint8_t* base_a = a.a_rows ? a.A : a.A + (int64_t)tile.m0 * a.lda;
    const uint8_t* base_b = a.B + (b_group(a, tile) + n0) * a.ldb;
    const int4v rsrcA = make_rsrc(base_a, (unsigned)(a.a_rows ? a.a_rows : min(C::BM, tile.m_end - tile.m0)) * (unsigned)a.lda);
    const int4v rsrcB = make_rsrc(base_b, (unsigned)min(C::BN, a.N - n0) * (unsigned)a.ldb);
    const int chunk = (lane & 7) ^ (4 * (wave & 1) + (lane >> 4));
    unsigned vo[C::LOADS];
#pragma unroll
    for (int j = 0; j < C::LOADS; ++j) {
        const int row = (j * C::NWAVES + wave) * 8 + (lane >> 3);
        if (row < C::BM) {
            const int r = row_of_a(a, tile.m0 + row, tile.m_end);
            vo[j] = r < 0 ? OOB : (unsigned)(a.a_rows ? r : row) * (unsigned)a.lda + chunk * 16;
        } else {
            const int r = row - C::BM;
            vo[j] = r >= C::BN || n0 + r >= a.N ? OOB : (unsigned)r * (unsigned)a.ldb + chunk * 16;
        }
    }
    const int ssize = byte ? 1 : 4;
    const char* base_sa = (const char*)a.SA + ((a.a_rows ? 0 : tile.m0) + kb0 * a.ldsa) * ssize;
    const char* base_sb = (const char*)a.SB + (B_BY_ROW ? n0 + kb0 * a.ldsb : sb_group(a, tile) + (int64_t)(n0 / kScaleBlock) * a.ldsb + kb0) * ssize;
    const int64_t step_sa = a.ldsa * ssize, step_sb = (B_BY_ROW ? a.ldsb : 1) * ssize;
    unsigned so[C::SLOADS];
#pragma unroll
    for (int j = 0; j < C::SLOADS; ++j) {
        const int i = j * C::NWAVES + wave;
        so[j] = OOB;
        if (i < C::SA_LOADS) {
            const int row = i * 64 + lane;
            const int r = row < C::BM ? row_of_a(a, tile.m0 + row, tile.m_end) : -1;
            if (r >= 0) so[j] = (unsigned)(a.a_rows ? r : row) * ssize;
        } else {
            const int r = (i - C::SA_LOADS) * 64 + lane;
            if (r < C::BN && n0 + r < a.N) so[j] = (unsigned)(B_BY_ROW ? r : (int64_t)(r / kScaleBlock) * a.ldsb) * ssize;
        }
    }
    const unsigned lds0 = __builtin_amdgcn_readfirstlane((int)lds_addr_of(lds));
    int kc = kb0;                                       // block copied next
    auto copy = [&](auto j_tag, unsigned stage) {
        constexpr int j = decltype(j_tag)::value;
        if constexpr (j < C::LOADS) {
            const bool of_a = (j * C::NWAVES + wave) * 8 < C::BM;
            copy16(of_a ? rsrcA : rsrcB, lds0 + stage + (j * C::NWAVES + wave) * 1024, vo[j], (unsigned)kc * kScaleBlock);
        } else {
            constexpr int s = j - C::LOADS;
            const int i = s * C::NWAVES + wave;
            const int4v r = make_rsrc(i < C::SA_LOADS ? base_sa : base_sb, kc < kb1 ? 0x7fffffffu : 0u);
            copy_scale<byte>(r, lds0 + stage + C::ROWS_BYTES + i * 256, so[s]);
        }
    };
    // Behind the last copy of a block: on to the next.  The last block of K may end inside: chunks past it are not copied, and blocks past the
    // last are zeros (both by an offset out of range), which keeps the number of copies in flight the same.
    auto next = [&]() {
        ++kc;
        base_sa += step_sa;
        base_sb += step_sb;
        if (kc >= kb1 || (kc + 1) * kScaleBlock > tile.k_end) {
#pragma unroll
            for (int j = 0; j < C::LOADS; ++j)
                if (kc * kScaleBlock + chunk * 16 >= tile.k_end) vo[j] = OOB;
        }
    };

    // fragments: chunks lg and lg + 4 of a row
    const int ra = wm + l16, rb = wn + l16;
    const int at_a = ra * 128 + ((lg ^ ((ra >> 1) & 7)) << 4), at_b = (C::BM + rb) * 128 + ((lg ^ ((rb >> 1) & 7)) << 4);
    const int at_sa = C::ROWS_BYTES + ra * 4, at_sb = C::ROWS_BYTES + C::SA_LOADS * 256 + (SUM == SUM_E8M0 ? rb : wn + 4 * lg) * 4;

    auto block = [&](const char* st, unsigned into) {
        Fragment<WIDE> fb[C::TN], fa[2];
        int ia[2] = {0, 0}, ib[C::TN];                  // scales as they lie: bits of a float, or a byte
        f4 sb[C::TN];
        auto read_a = [&](auto tm_tag) {
            constexpr int tm = decltype(tm_tag)::value;
            fa[tm & 1] = make_fragment<WIDE, A5>(*(const i4*)(st + at_a + tm * 2048), *(const i4*)(st + (at_a ^ 64) + tm * 2048));
            ia[tm & 1] = *(const int*)(st + at_sa + tm * 64);
        };
        auto value = [&](int raw) { return byte ? e8m0_value(raw) : __builtin_bit_cast(float, raw); };
        static_for<C::TN>([&](auto tn) {
            fb[tn] = make_fragment<WIDE, false>(*(const i4*)(st + at_b + tn * 2048), *(const i4*)(st + (at_b ^ 64) + tn * 2048));
            if constexpr (SUM == SUM_E8M0) {
                ib[tn] = *(const int*)(st + at_sb + tn * 64);
            } else if (B_BY_ROW || tn == 0) {
                const i4 raw = *(const i4*)(st + at_sb + tn * 64);
#pragma unroll
                for (int e = 0; e < 4; ++e) sb[tn][e] = value(raw[e]);
            }
        });
        read_a(ic<0>{});
        // Sums of a block wait DELAY tiles for their multiply-adds, so that those run under later instructions of the matrix cores.
        constexpr int TILES = C::TM * C::TN, DELAY = C::TN < 4 ? C::TN : 4;
        f4 p[DELAY];
        float scale_of[2];
        auto add = [&](auto i_tag) {
            constexpr int i = decltype(i_tag)::value, tm = i / C::TN, tn = i % C::TN;
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[tm][tn][e] += p[i % DELAY][e] * (B_BY_ROW ? scale_of[tm & 1] * sb[tn][e] : scale_of[tm & 1]);
            asm volatile("" : "+v"(acc[tm][tn]));       // here, not behind the last of the block's matrix instructions
        };
        static_for<TILES>([&](auto i_tag) {
            constexpr int i = decltype(i_tag)::value, tm = i / C::TN, tn = i % C::TN;
            if constexpr (tn == 0) {
                if constexpr (SUM != SUM_E8M0) scale_of[tm & 1] = B_BY_ROW ? value(ia[tm & 1]) : value(ia[tm & 1]) * sb[0][0];
                if constexpr (tm + 1 < C::TM) read_a(ic<tm + 1>{});
            }
            if constexpr (SUM == SUM_E8M0) {
                acc[tm][tn] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[tn].v, fa[tm & 1].v, acc[tm][tn], 0, A5 ? 1 : 0, 0, ib[tn], 0, ia[tm & 1]);
            } else {
                if constexpr (i >= DELAY) add(ic<i - DELAY>{});
                p[i % DELAY] = mma_block<A5>(fb[tn], fa[tm & 1], f4{0.f, 0.f, 0.f, 0.f});
            }
            constexpr int lo = i * C::ALL_LOADS / TILES, hi = (i + 1) * C::ALL_LOADS / TILES;
            static_for<hi - lo>([&](auto x) { copy(ic<lo + decltype(x)::value>{}, into); });
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (SUM != SUM_E8M0) static_for<DELAY>([&](auto x) { add(ic<TILES - DELAY + decltype(x)::value>{}); });
        next();
    };

    if (kb0 < kb1) {
        --kc;
        base_sa -= step_sa;
        base_sb -= step_sb;
        next();                                         // the first block may be the last
        static_for<C::STAGES - 1>([&](auto s) {
            static_for<C::ALL_LOADS>([&](auto j) { copy(j, decltype(s)::value * C::STAGE_BYTES); });
            next();
        });
        unsigned from = 0, into = (C::STAGES - 1) * C::STAGE_BYTES;
#pragma unroll 1
        for (int kb = kb0; kb < kb1; ++kb) {
            // this wave's copies of the block have landed; behind the barrier everybody's have, and nobody reads the block before
            wait_vmcnt<C::ALL_LOADS * (C::STAGES - 2)>();
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            if (kb == kb1 - 1 && (tile.k_end & 15)) {
                // K ends inside a 16-byte chunk: what lies past it is cleared in every row
                const int left = tile.k_end & (kScaleBlock - 1), c = left >> 4;
                for (int r = threadIdx.x; r < C::BM + C::BN; r += C::THREADS) {
                    u4* const p = (u4*)(lds + from + r * 128 + ((c ^ ((r >> 1) & 7)) << 4));
                    u4 v = *p;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int keep = (left & 15) - 4 * e;
                        v[e] &= keep >= 4 ? ~0u : keep <= 0 ? 0u : (1u << (8 * keep)) - 1;
                    }
                    *p = v;
                }
                __syncthreads();
            }
            block(lds + from, into);
            from = from + C::STAGE_BYTES == C::LOOP_BYTES ? 0 : from + C::STAGE_BYTES;
            into = into + C::STAGE_BYTES == C::LOOP_BYTES ? 0 : into + C::STAGE_BYTES;
        }
        wait_vmcnt<0>();
    }
    __syncthreads();
    if (a.splits > 1) {
        // The sums of this range of K go out as they lie in the lanes; the workgroup that arrives last at the tile adds all ranges in their order.
        typedef unsigned long long u64;
        u64* const planes = (u64*)(a.partial + (int64_t)blockIdx.x * a.splits * (C::BM * C::BN)) + threadIdx.x * 2;
        auto place = [&](int split, int i, int j) { return planes + ((int64_t)split * C::TM * C::TN + i * C::TN + j) * (C::THREADS * 2); };
        union Sums { f4 f; u64 u[2]; };
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int j = 0; j < C::TN; ++j) {
                Sums v;
                v.f = acc[i][j];
                store_agent(place(blockIdx.y, i, j), v.u[0]);
                store_agent(place(blockIdx.y, i, j) + 1, v.u[1]);
            }
        if (!last_to_arrive(a.counters + blockIdx.x, a.splits, (int*)lds, threadIdx.x == 0)) return;
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int j = 0; j < C::TN; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
        for (int s = 0; s < a.splits; ++s)
#pragma unroll
            for (int i = 0; i < C::TM; ++i)
#pragma unroll
                for (int j = 0; j < C::TN; ++j) {
                    Sums v;
                    v.u[0] = load_agent(place(s, i, j));
                    v.u[1] = load_agent(place(s, i, j) + 1);
                    acc[i][j] += v.f;
                }
        __syncthreads();
    }
    store_tile<C, WIDE>(lds, a, tile, n0, [&](auto&& put) {
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int j = 0; j < C::TN; ++j) put(wm + i * 16 + l16, wn + j * 16 + 4 * lg, acc[i][j]);
    });
}

}  // namespace hgemm
