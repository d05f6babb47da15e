// The host side of the feed-forward block's operators with every launch written
// down instead: built for the CPU alone by test_block_launches.py.  Pointers are
// never followed.
#include "../paper_2512_08365_amd/csrc/block.hip"

#include <stdarg.h>
#include <stdio.h>

#include <string>

namespace {

std::string g_log, g_error;

void note(const char* fmt, ...)
{
    char line[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(line, sizeof(line), fmt, ap);
    va_end(ap);
    g_log += line;
    g_log += '\n';
}

hipError_t product(const char* what, const mag::Mm& p, int kind, int tile)
{
    note("what=%s kind=%d tile=%d a_ld=%lld a_mc=%d b_ld=%lld b_mc=%d R=%lld S=%lld K=%lld batch=%d "
         "splits=%d symmetric=%d scale=%.9g mix=%.9g diagonal=%.9g mixed=%d",
         what, kind, tile, (long long)p.a.ld, p.a.mc, (long long)p.b.ld, p.b.mc, (long long)p.R,
         (long long)p.S, (long long)p.K, p.batch, p.splits, p.symmetric, p.o.scale, p.o.mix, p.o.diagonal,
         p.o.m != nullptr);
    return hipSuccess;
}

}  // namespace

namespace mag {

int set_error(int code, const char* msg)
{
    g_error = msg;
    return code;
}
int set_hip_error(hipError_t, const char* where) { return set_error(MAG_E_HIP, where); }
void clear_error() { g_error.clear(); }
int device_cu_count() { return 256; }

hipError_t launch_mm_bf16(const Mm& p, int tile, hipStream_t) { return product("linear", p, MM_BF16, tile); }
hipError_t launch_mm_f16(const Mm& p, int tile, hipStream_t) { return product("linear", p, MM_F16, tile); }
hipError_t launch_mm_f32(const Mm& p, hipStream_t) { return product("linear", p, MM_F32, TILE_64); }
hipError_t launch_mm_f32_parts(const Mm& p, int tile, hipStream_t)
{
    return product("linear", p, MM_F32_PARTS, tile);
}
hipError_t launch_mm_partial(const Mm& p, int kind, int tile, hipStream_t)
{
    return product("partial", p, kind, tile);
}
hipError_t launch_mm_orth(const Mm& p, int tile, hipStream_t) { return product("update", p, MM_HALVES, tile); }
hipError_t launch_mm_two(const Mm& dx, const Mm& dw, int kind, int, int, hipStream_t)
{
    (void)product("two", dx, kind, TILE_64);
    return product("two", dw, kind, TILE_64);
}
hipError_t launch_mm_join(const Mm&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_orth_join(const Mm&, hipStream_t) { return hipSuccess; }
hipError_t launch_skinny(const SkinnyParams& p, int dtype, hipStream_t)
{
    note("what=skinny kind=%d across=%d M=%lld N=%lld K=%lld", dtype, p.across, (long long)p.M,
         (long long)p.N, (long long)p.K);
    return hipSuccess;
}
hipError_t launch_prepare(const PackParams* a, const PackParams* b, const ColumnSums*, int kind, hipStream_t)
{
    for (const PackParams* p : {a, b})
        if (p)
            note("what=pack kind=%d rows=%lld cols=%lld rs=%lld cs=%lld ld=%lld", kind, (long long)p->rows,
                 (long long)p->cols, (long long)p->rs, (long long)p->cs, (long long)p->ld);
    return hipSuccess;
}
int64_t slope_chunks(int64_t, int64_t) { return 1; }
hipError_t launch_slope(const SlopeParams&, int, hipStream_t) { return hipSuccess; }
int norm_parts(int64_t, int64_t, int) { return 1; }
hipError_t launch_norm(const NormParams&, int, int, hipStream_t) { return hipSuccess; }
hipError_t launch_norm_backward(const NormParams&, int, int, hipStream_t) { return hipSuccess; }
hipError_t launch_orth_begin(const OrthParams& p, int, hipStream_t)
{
    note("what=begin scale=%.9g", p.scale);
    return hipSuccess;
}

}  // namespace mag

extern "C" const char* launches() { return g_log.c_str(); }
extern "C" void clear_launches() { g_log.clear(); }
extern "C" const char* last_error() { return g_error.c_str(); }
