// Host side of the products of 8-bit floats: checks, the choice of a kernel, launches.
#include "scaled_kernels.hpp"
#include "scaled_tile.hpp"          // SUM_*

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <new>
#include <string>
#include <vector>

using namespace hgemm;

namespace {

const std::vector<ScaledEntry>& entries()
{
    static const std::vector<ScaledEntry> all = [] {
        std::vector<ScaledEntry> v;
        add_scaled_entries_0(v);
        add_scaled_entries_1(v);
        add_scaled_entries_2(v);
        add_scaled_entries_3(v);
        add_scaled_entries_4(v);
        return v;
    }();
    return all;
}

enum Family { FAMILY_EMPTY, FAMILY_ROWS, FAMILY_TILE, FAMILY_PHASED };

struct Choice {
    Family family = FAMILY_TILE;
    int bm = 0, bn = 0, st = 0, wv = 0, gm = 0, sk = 1;
    const ScaledEntry* entry = nullptr;
};

int sum_of(const ScaledArgs& a) { return a.c_type == HGEMM_F32 ? a.e8m0 ? SUM_WIDE_E8M0 : SUM_WIDE : a.e8m0 ? SUM_E8M0 : SUM_SCALED; }

// The compiled kernel that a choice names (st or wv = 0: any) and that has the sums of the problem.
const ScaledEntry* find_entry(const ScaledArgs& a, hgemm_byte_t a_type, const Choice& c)
{
    if (c.family == FAMILY_PHASED && a.K % 16) return nullptr;      // does not clear what lies past K in a 16-byte chunk
    for (const ScaledEntry& e : entries()) {
        const Family f = e.bn == 16 ? FAMILY_ROWS : e.st == 0 ? FAMILY_PHASED : FAMILY_TILE;
        if (f == c.family && e.bm == c.bm && e.bn == c.bn && (!c.st || e.st == c.st) && (!c.wv || e.wm * e.wn == c.wv) && e.kernel[sum_of(a)][a_type][a.b_by_row]) return &e;
    }
    return nullptr;
}

// Microseconds of one workgroup for a block of K: alone on its compute unit (its own chain of waits), and its share of a unit that `resident` of
// them fill.  Measured with f32 scales and a 16-bit C: one tile a unit, K of 2048 and 8192 (alone); 4001 x 14336 x 4096 (full).
// Of 60 problems drawn at random (their timings are among the profiles) the pick was within 5 % of the fastest of all kernels on 38 and within 15 % on 50, in the mean
// 7 % behind it.  Furthest: 29 rows of A where a long K meets few columns (192 x 6528: 11.8 us streaming, 6.8 with K split in eight), and groups padded to
// 128 rows of which most are empty (79 x 8 of 60 experts 1.3), where a plan knows the rows there is room for and not those there are.
struct Speed {
    Family family;
    int bm, bn, resident;
    double alone, full;
};
const Speed speeds[] = {
    {FAMILY_TILE, 16, 64, 3, 0.217, 0.115}, {FAMILY_TILE, 32, 64, 3, 0.255, 0.136}, {FAMILY_TILE, 64, 64, 3, 0.30, 0.183}, {FAMILY_TILE, 32, 128, 2, 0.311, 0.220},
    {FAMILY_TILE, 64, 128, 2, 0.379, 0.309}, {FAMILY_TILE, 128, 128, 2, 0.734, 0.495}, {FAMILY_TILE, 256, 128, 1, 0.958, 0.958}, {FAMILY_TILE, 256, 256, 1, 1.62, 1.62},
    {FAMILY_PHASED, 128, 128, 2, 0.561, 0.485}, {FAMILY_PHASED, 256, 256, 1, 1.50, 1.50},
};

// Predicted microseconds of a kernel: the longest of its workgroups' rounds over the compute units, and memory at what streaming kernels reach.
// A split of K costs its sums' way to memory and back.  Only the order of the predictions matters.
double predict(const ScaledArgs& a, const Speed& s, int splits)
{
    const double M = a.M, N = a.N, K = a.K, units = (double)compute_units();
    const bool rows = a.group == HGEMM_GROUPS_ROWS, depth = a.group == HGEMM_GROUPS_DEPTH;
    const double used = rows ? std::min<double>(a.groups, M) : 1, deep = depth ? a.groups : 1;
    // groups of rows end inside a tile: half a tile each, and a tile at least
    const double tiles_m = rows ? std::max(used, M / s.bm + used * 0.5) : ceil(M / s.bm);
    const double tiles = tiles_m * ceil(N / s.bn) * deep, work = tiles * splits;
    const double blocks = std::max(1.0, ceil(ceil(K / deep / kScaleBlock) / splits));
    const bool wide = a.c_type == HGEMM_F32;
    const double full = s.full * (wide ? 1.9 : a.e8m0 ? 0.9 : 1);
    const double alone = wide ? std::max(s.alone * 1.3, full) : s.alone * (a.e8m0 && s.family == FAMILY_PHASED ? 0.85 : 1);
    const double a_round = units * s.resident, rounds = floor(work / a_round), left = ceil((work - rounds * a_round) / units);
    const double size = s.bm * s.bn / 65536.0, each = 0.7 + 6.5 * size + rows;     // start and end of a tile; a look for its group
    double t = 2.2 + rounds * (blocks * std::max(alone, s.resident * full) + each);
    if (left > 0) t += blocks * std::max(alone, work > units ? left * full : 0) + each;
    const double bytes = M * K + used * N * K + M * N * deep * (wide ? 4 : 2);
    t = std::max(t, 3.5 + bytes / 5.2e6);
    if (splits > 1) t += 1 + work * s.bm * s.bn * 8 / 2e6;
    return t;
}

// Few rows of A, B streamed into registers: what they reach of memory (16 rows of A or 32 a workgroup).  Not with groups: their
// workgroups, one to a group and 16 rows of B, are too many (24 x 4 rows of 32 experts, 4096 x 2048: 58 us, tiles 44).
double predict_rows(const ScaledArgs& a, int bm)
{
    return 2.8 + ((double)a.N * a.K + (double)a.M * a.N * 2) / (bm == 16 ? 3.6e6 : 2.2e6);
}

void choose(const ScaledArgs& a, hgemm_byte_t a_type, Choice& c)
{
    double best = 1e300;
    for (int bm = 16; bm <= 32; bm *= 2) {
        if (a.M > bm || a.group != HGEMM_GROUPS_NONE) continue;
        const double t = predict_rows(a, bm);
        if (t >= best) continue;
        best = t;
        const int64_t blocks = blocks_of(a.K);
        c = Choice{};
        c.family = FAMILY_ROWS;
        c.bm = bm;
        c.bn = 16;
        c.wv = blocks >= 64 ? 16 : blocks >= 16 ? 8 : 4;
    }
    for (const Speed& s : speeds) {
        Choice t;
        t.family = s.family;
        t.bm = s.bm;
        t.bn = s.bn;
        if (!find_entry(a, a_type, t)) continue;
        const int most = s.family == FAMILY_TILE && a.group == HGEMM_GROUPS_NONE ? 16 : 1;
        for (t.sk = 1; t.sk <= most; t.sk *= 2) {
            if (t.sk > 1 && blocks_of(a.K) < 4 * t.sk) break;
            const double us = predict(a, s, t.sk);
            if (us < best) { best = us; c = t; }
        }
    }
}

// "rows,bm=..,bn=16[,wv=..]", "tile,bm=..,bn=..[,st=..][,wv=..][,gm=..][,sk=..]" or "phased,bm=..,bn=..[,wv=..][,gm=..]"
bool parse(const char* spec, Choice& c)
{
    const char* const names[] = {"rows", "tile", "phased"};
    const Family families[] = {FAMILY_ROWS, FAMILY_TILE, FAMILY_PHASED};
    const char* p = nullptr;
    for (int i = 0; i < 3; ++i)
        if (!strncmp(spec, names[i], strlen(names[i]))) {
            c.family = families[i];
            p = spec + strlen(names[i]);
        }
    if (!p) return false;
    while (*p) {
        if (p[0] != ',' || !p[1] || !p[2] || p[3] != '=') return false;
        char* end;
        const long v = strtol(p + 4, &end, 10);
        if (end == p + 4 || v < 0 || v > 1024) return false;
        if (!strncmp(p + 1, "bm", 2)) c.bm = (int)v;
        else if (!strncmp(p + 1, "bn", 2)) c.bn = (int)v;
        else if (!strncmp(p + 1, "st", 2)) c.st = (int)v;
        else if (!strncmp(p + 1, "wv", 2)) c.wv = (int)v;
        else if (!strncmp(p + 1, "gm", 2)) c.gm = (int)v;
        else if (!strncmp(p + 1, "sk", 2) && c.family == FAMILY_TILE && v) c.sk = (int)v;
        else return false;
        p = end;
    }
    return true;
}

}  // namespace

struct hgemm_scaled_plan_s {
    ScaledArgs args;
    Choice choice;
    void (*kernel)(ScaledArgs) = nullptr;
    int64_t grid_x = 0, grid_y = 1;
    void* workspace = nullptr;
    size_t workspace_bytes = 0;
    bool clearing = false;      // the counters may still be on their way to zero
};

namespace {

// Fills the arguments from the description; the pointers come with the run.
hgemm_status_t describe_problem(ScaledArgs& a, int64_t M, int64_t N, int64_t K, const hgemm_scaled_t& d)
{
    const int64_t most = (int64_t)1 << 23;
    if (M < 0 || N < 0 || K < 0) return HGEMM_ERR_INVALID_ARG;
    if ((unsigned)d.a > HGEMM_E5M2 || (unsigned)d.c > HGEMM_F32 || (unsigned)d.scale > HGEMM_SCALE_E8M0 || (unsigned)d.group > HGEMM_GROUPS_DEPTH) return HGEMM_ERR_INVALID_ARG;
    if (d.b_block_rows != 1 && d.b_block_rows != kScaleBlock) return HGEMM_ERR_INVALID_ARG;
    const bool grouped = d.group != HGEMM_GROUPS_NONE;
    if (grouped ? d.groups < 1 || d.groups > 1024 : d.groups != 0) return HGEMM_ERR_INVALID_ARG;
    if (d.a_rows < 0 || (d.a_rows && d.group != HGEMM_GROUPS_ROWS)) return HGEMM_ERR_INVALID_ARG;
    const bool by_row = d.b_block_rows == 1;
    if (by_row && d.group == HGEMM_GROUPS_ROWS) return HGEMM_ERR_UNSUPPORTED;
    const int64_t lda = d.lda ? d.lda : round_up(K, 16), ldb = d.ldb ? d.ldb : round_up(K, 16), ldc = d.ldc ? d.ldc : N;
    const int64_t rows_a = d.a_rows ? d.a_rows : M;
    const int64_t ldsa = d.ld_scale_a ? d.ld_scale_a : rows_a, ldsb = d.ld_scale_b ? d.ld_scale_b : by_row ? N : blocks_of(K);
    if (lda < K || ldb < K || ldc < N || ldsa < rows_a || ldsb < (by_row ? N : blocks_of(K))) return HGEMM_ERR_INVALID_ARG;
    if (lda % 16 || ldb % 16) return HGEMM_ERR_UNSUPPORTED;
    if (lda >= most || ldb >= most || M > 0x7fffff00LL || N > 0x7fffff00LL || rows_a > 0x7fffff00LL) return HGEMM_ERR_UNSUPPORTED;
    if (!by_row && ldsb >= (int64_t)1 << 28) return HGEMM_ERR_UNSUPPORTED;
    if (N * ldb > 0x7fffffffLL || (d.a_rows && rows_a * lda > 0x7fffffffLL)) return HGEMM_ERR_UNSUPPORTED;
    a = ScaledArgs{};
    a.M = (int)M; a.N = (int)N; a.K = (int)K;
    a.lda = (int)lda; a.ldb = (int)ldb;
    a.ldc = ldc; a.ldsa = ldsa; a.ldsb = ldsb;
    a.a_rows = (int)d.a_rows;
    a.groups = d.groups; a.group = d.group;
    a.b_by_row = by_row; a.e8m0 = d.scale == HGEMM_SCALE_E8M0; a.c_type = d.c;
    return HGEMM_OK;
}

// The most row tiles of `bm` rows that any offsets can give: a tile more for each group and one for the rows behind them.
int64_t most_row_tiles(const ScaledArgs& a, int64_t bm)
{
    if (a.group != HGEMM_GROUPS_ROWS) return hgemm_tiles(a.M, bm);
    const int64_t t = a.M / bm + a.groups + 1;
    return t < a.M ? t : a.M;
}

hgemm_status_t make_plan_unguarded(hgemm_scaled_plan_t* out, int64_t M, int64_t N, int64_t K, const hgemm_scaled_t* desc, const char* spec)
{
    if (!out || !desc) return HGEMM_ERR_INVALID_ARG;
    ScaledArgs a;
    hgemm_status_t st = describe_problem(a, M, N, K, *desc);
    if (st != HGEMM_OK) return st;
    Choice c;
    if (spec) {
        if (!parse(spec, c)) return HGEMM_ERR_INVALID_ARG;
    } else {
        choose(a, desc->a, c);
    }
    if (!M || !N) c.family = FAMILY_EMPTY;
    if (c.family != FAMILY_EMPTY) {
        c.entry = find_entry(a, desc->a, c);
        if (!c.entry) return HGEMM_ERR_UNSUPPORTED;
        c.st = c.entry->st;
        c.wv = c.entry->wm * c.entry->wn;
    }
    if (c.family != FAMILY_EMPTY && !current_device_is_gfx950()) return HGEMM_ERR_ARCH;
    hgemm_scaled_plan_s* p = new (std::nothrow) hgemm_scaled_plan_s;
    if (!p) return HGEMM_ERR_ALLOC;
    // Rows of tiles that share columns of B; a group that has one row of tiles shares nothing, and then whole rows one after another stream better
    // (24 x 4 rows of 32 experts of 4096 x 2048: 43.6 us, by eight rows 48.1; 128 x 4: 49.9 and 54.8; 8 x 2 of 8, 14336 x 4096: 75 and 72).
    if (!c.gm) c.gm = a.group == HGEMM_GROUPS_ROWS && M <= (int64_t)c.bm * a.groups ? 1 : 8;
    p->args = a;
    p->choice = c;
    if (c.family != FAMILY_EMPTY) {
        ScaledArgs& g = p->args;
        g.tiles_m = (int)most_row_tiles(a, c.bm);
        g.tiles_n = (int)hgemm_tiles(N, c.bn);
        g.swizzle = c.gm < g.tiles_m ? c.gm : g.tiles_m;
        set_tile_map(g);
        p->grid_x = (int64_t)g.tiles_m * g.tiles_n;
        p->grid_y = a.group == HGEMM_GROUPS_DEPTH ? a.groups : 1;
        p->kernel = c.entry->kernel[sum_of(a)][desc->a][a.b_by_row];
        g.splits = 1;
        const int64_t blocks = blocks_of(K);
        if (c.sk > 1 && blocks > 1 && a.group == HGEMM_GROUPS_NONE) {
            const int64_t each = (blocks + c.sk - 1) / c.sk;
            g.splits = (int)((blocks + each - 1) / each);       // no range is empty
            g.k_per_split = (int)(each * kScaleBlock);
        }
        p->choice.sk = g.splits;
        if (p->grid_x >= (1 << 24) || !fits_grid(p->grid_x, c.entry->threads)) { delete p; return HGEMM_ERR_UNSUPPORTED; }
        if (c.entry->lds_bytes && hipFuncSetAttribute((const void*)p->kernel, hipFuncAttributeMaxDynamicSharedMemorySize, c.entry->lds_bytes) != hipSuccess) {
            (void)hipGetLastError();
            delete p;
            return HGEMM_ERR_LAUNCH;
        }
        if (g.splits > 1) {
            const size_t counters = round_up(p->grid_x * sizeof(int), 256);
            p->grid_y = g.splits;
            p->workspace_bytes = counters + (size_t)p->grid_x * g.splits * c.bm * c.bn * sizeof(float);
            if (hipMalloc(&p->workspace, p->workspace_bytes) != hipSuccess || hipMemset(p->workspace, 0, counters) != hipSuccess) {
                (void)hipGetLastError();
                if (p->workspace) (void)hipFree(p->workspace);
                delete p;
                return HGEMM_ERR_ALLOC;
            }
            g.counters = (int*)p->workspace;
            p->clearing = true;
            g.partial = (float*)((char*)p->workspace + counters);
        }
    }
    *out = p;
    return HGEMM_OK;
}

hgemm_status_t make_plan(hgemm_scaled_plan_t* out, int64_t M, int64_t N, int64_t K, const hgemm_scaled_t* desc, const char* spec)
{
    try {
        return make_plan_unguarded(out, M, N, K, desc, spec);
    } catch (...) {                                     // the list of kernels could not be allocated
        return HGEMM_ERR_ALLOC;
    }
}

}  // namespace

extern "C" {

hgemm_status_t hgemm_scaled_plan(hgemm_scaled_plan_t* out, int64_t M, int64_t N, int64_t K, const hgemm_scaled_t* desc)
{
    return make_plan(out, M, N, K, desc, nullptr);
}

hgemm_status_t hgemm_scaled_plan_override(hgemm_scaled_plan_t* out, int64_t M, int64_t N, int64_t K, const hgemm_scaled_t* desc, const char* spec)
{
    return spec ? make_plan(out, M, N, K, desc, spec) : HGEMM_ERR_INVALID_ARG;
}

hgemm_status_t hgemm_scaled_run(hgemm_scaled_plan_t plan, const void* A, const void* scale_a, const void* B, const void* scale_b, void* C, const int32_t* offsets,
                                const int32_t* index, void* hip_stream)
{
    if (!plan) return HGEMM_ERR_INVALID_ARG;
    if (plan->choice.family == FAMILY_EMPTY) return HGEMM_OK;
    ScaledArgs a = plan->args;
    if (!C || (a.K && (!A || !B || !scale_a || !scale_b))) return HGEMM_ERR_INVALID_ARG;
    if ((a.group && !offsets) || (a.a_rows && !index)) return HGEMM_ERR_INVALID_ARG;
    const size_t elem = type_size((hgemm_type_t)a.c_type), scale = a.e8m0 ? 1 : 4;
    if (!aligned(A, 16) || !aligned(B, 16) || !aligned(scale_a, scale) || !aligned(scale_b, scale) || !aligned(C, elem) || !aligned(offsets, 4) || !aligned(index, 4))
        return HGEMM_ERR_INVALID_ARG;
    a.A = (const uint8_t*)A;
    a.B = (const uint8_t*)B;
    a.SA = scale_a;
    a.SB = scale_b;
    a.C = C;
    a.offsets = offsets;
    a.index = index;
    const dim3 grid((unsigned)plan->grid_x, (unsigned)plan->grid_y);
    const hipStream_t stream = (hipStream_t)hip_stream;
    if (!wait_for_clearing(plan->clearing, stream)) return HGEMM_ERR_LAUNCH;
    const ScaledEntry& e = *plan->choice.entry;
    plan->kernel<<<grid, e.threads, e.lds_bytes, stream>>>(a);
    return hipGetLastError() == hipSuccess ? HGEMM_OK : HGEMM_ERR_LAUNCH;
}

hgemm_status_t hgemm_scaled_destroy(hgemm_scaled_plan_t plan)
{
    if (!plan) return HGEMM_OK;
    if (plan->workspace && hipFree(plan->workspace) != hipSuccess) (void)hipGetLastError();
    delete plan;
    return HGEMM_OK;
}

size_t hgemm_scaled_workspace_bytes(hgemm_scaled_plan_t plan) { return plan ? plan->workspace_bytes : 0; }

hgemm_status_t hgemm_scaled_describe(hgemm_scaled_plan_t plan, char* buf, size_t n)
{
    if (!plan || !buf || n == 0) return HGEMM_ERR_INVALID_ARG;
    const Choice& c = plan->choice;
    char s[96];
    if (c.family == FAMILY_EMPTY) snprintf(s, sizeof s, "empty");
    else if (c.family == FAMILY_ROWS) snprintf(s, sizeof s, "rows,bm=%d,bn=%d,wv=%d", c.bm, c.bn, c.wv);
    else if (c.family == FAMILY_PHASED) snprintf(s, sizeof s, "phased,bm=%d,bn=%d,wv=%d,gm=%d", c.bm, c.bn, c.wv, c.gm);
    else snprintf(s, sizeof s, "tile,bm=%d,bn=%d,st=%d,wv=%d,gm=%d,sk=%d", c.bm, c.bn, c.st, c.wv, c.gm, c.sk);
    if (strlen(s) + 1 > n) { buf[0] = '\0'; return HGEMM_ERR_INVALID_ARG; }
    strcpy(buf, s);
    return HGEMM_OK;
}

}  // extern "C"
