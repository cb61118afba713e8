// Layout of the backward over a source stack in 8 or 4 bits, its workspace, and
// its launch.  Host code only.
#include <algorithm>

#include "cache_bwd.h"

namespace lrar {

namespace {

// Tokens up to which the low-rank backward splits each token's sources over a
// workgroup.  Split / not, gradient rows: e4m3, 49 sources, d = 1024: 700 tokens 28 /
// 38 us, 1001 tokens 36 / 43, 1500 tokens 56 / 56, 2500 tokens 90 / 81; e2m1, 30
// sources, d = 512: 1001 tokens 24 / 35, 2500 tokens 50 / 43.  Deferred: e4m3, 49
// sources: 600 tokens 19 / 22, 1001 tokens 20 / 22, 1500 tokens 27 / 24.
constexpr int64_t kSplitBwd = 1024;
// Waves from which a group takes several tokens (as in the forward), and the
// sources up to which their statistics fit LDS.
constexpr int64_t kManyWaves = 2048, kManySources = 128;
// Workgroups from which one of full-rank keys takes two or four tokens in turn, for
// fewer rows of dq partials: e2m1, 49 x 2048 x 1024: four tokens 89 us, two 94, one 97
// (the sum over the rows alone 5, 9 and 15).
constexpr int64_t kFullBlocks = 512;

}  // namespace

CacheBwdPlan cache_bwd_plan(const CacheProblem &p)
{
    CacheBwdPlan pl;
    const bool full = p.mode == LRAR_MODE_FULL;
    const int64_t units = cache_blocks(p.d) * (p.format == LRAR_CACHE_FP8 ? 2 : 1);
    const int64_t groups = units <= 16 ? 4 : units <= 32 ? 2 : 1;  // of lanes in a wave
    const int many = bwd_many(p.d);
    pl.split = !full && p.N <= kSplitBwd;
    pl.many = !full && !pl.split && p.S <= kManySources && p.N >= kManyWaves * groups * many;
    pl.tpw = !full ? 1 : p.N >= 4 * kFullBlocks ? 4 : p.N >= 2 * kFullBlocks ? 2 : 1;
    const int64_t per = full ? pl.tpw : pl.split ? 1 : kWaves * groups * (pl.many ? many : 1);
    pl.nblocks = (int)((p.N + per - 1) / per);
    return pl;
}

// The dq partials (rows of the most sources, which take the fewest tokens a
// workgroup), and the weights [S][N] of a low-rank backward that writes gradient
// rows.  Grows with S: a buffer sized for the deepest site of a pass serves all.
namespace {

size_t partial_bytes(const CacheProblem &p)
{
    CacheProblem q = p;
    q.S = std::max(p.S, kManySources + 1);
    return ((size_t)cache_bwd_plan(q).nblocks * (size_t)p.r * sizeof(float) + 15) / 16 * 16;
}

}  // namespace

size_t cache_bwd_workspace_bytes(const CacheProblem &p)
{
    const bool weights = p.mode != LRAR_MODE_FULL && !cache_bwd_plan(p).split;
    return partial_bytes(p) + (weights ? (size_t)p.S * (size_t)p.N * sizeof(float) : 0);
}

int launch_cache_bwd(const CacheProblem &p, const void *dH, void *dV, void *dK, float *coef,
                     float *dq, void *ws, bool accumulate, hipStream_t st, std::string *err)
{
    float *partial = static_cast<float *>(ws);
    const bool deferred = coef != nullptr;
    if (!deferred)
        coef = partial + partial_bytes(p) / sizeof(float);
    hipError_t e = hipSuccess;
    if (p.N > 0)
        e = p.format == LRAR_CACHE_FP8
                ? launch_cache_bwd_fp8(p, dH, dV, dK, coef, deferred, partial, accumulate, st)
                : launch_cache_bwd_fp4(p, dH, dV, dK, coef, deferred, partial, accumulate, st);
    if (e == hipSuccess)
        e = launch_dq_reduce(partial, dq, p.N > 0 ? cache_bwd_plan(p).nblocks : 0, (int)p.r,
                             accumulate, st);
    return hip_status(e, "cache_route_bwd launch", err);
}

}  // namespace lrar
