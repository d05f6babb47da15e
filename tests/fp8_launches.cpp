// The host side of the 8-bit operators with every launch written down instead:
// built for the CPU alone by test_fp8_launches.py.  Pointers are never followed.
#include "../paper_2512_08365_amd/csrc/fp8.hip"

#include <stdarg.h>
#include <stdio.h>

#include <string>

namespace {

std::string g_log, g_error;

void note(const char* fmt, ...)
{
    char line[1024];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(line, sizeof(line), fmt, ap);
    va_end(ap);
    g_log += line;
    g_log += '\n';
}

hipError_t product(const char* what, int tile, const mag::Mm8& p, int dtype)
{
    note("what=%s tile=%d a=%llu lda=%lld b=%llu ldb=%lld R=%lld S=%lld K=%lld sa=%llu sa_cs=%lld sb=%llu sb_cs=%lld "
         "by_row=%d splits=%d partial=%llu partial_ld=%lld dtype=%d",
         what, tile, (unsigned long long)p.a, (long long)p.lda, (unsigned long long)p.b, (long long)p.ldb,
         (long long)p.R, (long long)p.S, (long long)p.K, (unsigned long long)p.sa.p, (long long)p.sa.cs,
         (unsigned long long)p.sb.p, (long long)p.sb.cs, p.by_row, p.splits, (unsigned long long)p.partial,
         (long long)p.partial_ld, dtype);
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

hipError_t launch_quantize(const QuantizeParams&, int, int, bool, hipStream_t) { return hipSuccess; }
hipError_t launch_mm8_64(const Mm8& p, int dtype, hipStream_t) { return product("tiles", TILE_64, p, dtype); }
hipError_t launch_mm8_128(const Mm8& p, int dtype, hipStream_t) { return product("tiles", TILE_128, p, dtype); }
hipError_t launch_mm8_256(const Mm8& p, int dtype, hipStream_t) { return product("tiles", TILE_256, p, dtype); }
hipError_t launch_skinny8(const Mm8& p, int dtype, hipStream_t) { return product("skinny", TILE_64, p, dtype); }
hipError_t launch_pack8(const Pack8Params& p, hipStream_t)
{
    note("what=pack src=%llu rs=%lld cs=%lld rows=%lld cols=%lld dst=%llu ld=%lld", (unsigned long long)p.src,
         (long long)p.rs, (long long)p.cs, (long long)p.rows, (long long)p.cols, (unsigned long long)p.dst,
         (long long)p.ld);
    return hipSuccess;
}
hipError_t launch_mm_join(const Mm& p, int dtype, hipStream_t)
{
    note("what=join R=%lld S=%lld splits=%d partial=%llu partial_ld=%lld dtype=%d", (long long)p.R, (long long)p.S,
         p.splits, (unsigned long long)p.partial, (long long)p.partial_ld, dtype);
    return hipSuccess;
}

}  // namespace mag

extern "C" const char* launches() { return g_log.c_str(); }
extern "C" void clear_launches() { g_log.clear(); }
extern "C" const char* last_error() { return g_error.c_str(); }
