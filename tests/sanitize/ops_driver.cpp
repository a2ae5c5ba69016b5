// ops_driver.cpp -- drives the checks of include/dsim_ops.h's entry points over
// random and extreme arguments; launches are replaced by stand-ins.
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "../../paper_2111_05426_amd/csrc/ops.h"

namespace dsim {
static long launches;
dsim_status fail(dsim_status st, const char *fmt, ...)
{
    char text[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text, sizeof text, fmt, ap);
    va_end(ap);
    return st;
}
dsim_status launch_append(const AppendArgs &, hipStream_t) { return ++launches, DSIM_OK; }
size_t attend_workspace(int32_t q, int32_t h, int32_t d) { return (size_t)(q / h) * (size_t)d * 64; }
dsim_status launch_attend(const AttendArgs &, hipStream_t) { return ++launches, DSIM_OK; }
dsim_status launch_logits(const dsim_logits &, hipStream_t) { return ++launches, DSIM_OK; }
}  // namespace dsim

static uint64_t g_state = 1;
static uint64_t rnd()
{
    uint64_t z = (g_state += 0x9e3779b97f4a7c15ull);
    z = (z ^ (z >> 30)) * 0xbf58476d1ce4e5b9ull;
    z = (z ^ (z >> 27)) * 0x94d049bb133111ebull;
    return z ^ (z >> 31);
}

// mostly `usual`, sometimes an extreme
static int64_t odd64(int64_t usual)
{
    static const int64_t v[] = {0, 1, -1, 15, 16, 1 << 20, (1 << 20) + 1, INT32_MAX, (int64_t)INT32_MAX + 1, INT64_MAX,
                                INT64_MIN, (int64_t)1 << 61, ((int64_t)1 << 62) + 16};
    return rnd() % 24 ? usual : v[rnd() % (sizeof v / sizeof *v)];
}
static int32_t odd32(int32_t usual)
{
    static const int32_t v[] = {0, 1, -1, 7, 16, 256, 257, 4096, 4097, 1 << 20, 1 << 30, INT32_MAX, INT32_MIN};
    return rnd() % 24 ? usual : v[rnd() % (sizeof v / sizeof *v)];
}
static char *ptr() { return rnd() % 40 ? (char *)4096 : rnd() % 2 ? nullptr : (char *)4097; }

int main()
{
    long ok = 0, refused = 0;
    for (int i = 0; i < 300000; ++i) {
        const int es = (int)(rnd() % 4);
        dsim_kv_cache c{};
        c.k = ptr(), c.v = ptr(), c.block_table = (const int32_t *)ptr();
        if (rnd() % 8 == 0) c.k_scale = (const float *)ptr();
        c.n_pages = odd64(8), c.page_stride = odd64(4096), c.slot_stride = odd64(64), c.head_stride = odd64(1024);
        c.table_stride = odd64(4), c.dtype = odd32(es), c.n_heads = odd32(4), c.head_dim = odd32(64);
        c.page_size = odd32(16), c.n_seq = odd32(3), c.table_width = odd32(4);
        dsim_rows r[4];
        for (auto &x : r) x = {ptr(), odd64(1024), odd64(64)};
        const int32_t dtype = odd32(es == 3 ? 1 : es), rot = odd32(64), heads = odd32(8);
        dsim_status st = dsim_kv_append(rnd() % 99 ? &c : nullptr, odd64(5), dtype, &r[0], &r[1], rnd() % 2 ? &r[2] : nullptr,
                                        rnd() % 2 ? &r[3] : nullptr, heads, (const int32_t *)ptr(), (const int32_t *)ptr(),
                                        (const float *)ptr(), odd64(99), rot, odd32(0), nullptr, nullptr);
        st == DSIM_OK ? ++ok : ++refused;
        const size_t ws = dsim_paged_attention_workspace(odd32(8), odd32(4), odd32(64));
        st = dsim_paged_attention(&c, dtype, &r[0], &r[3], heads, (const int32_t *)ptr(), rnd() % 50 ? 0.1f : 1.0f / 0.0f,
                                  odd32(0), nullptr, nullptr, ptr(), rnd() % 9 ? ws : (size_t)odd64(0), nullptr);
        st == DSIM_OK ? ++ok : ++refused;
        dsim_logits a{};
        a.logits = ptr(), a.out = ptr(), a.logits_stride = odd64(100), a.out_stride = odd64(100), a.n_rows = odd64(3);
        a.vocab = odd32(100), a.dtype = odd32((int32_t)(rnd() % 3)), a.history_stride = odd64(9), a.history_width = odd32(9);
        if (rnd() % 2) a.history = (const int32_t *)ptr(), a.history_len = (const int32_t *)ptr(), a.repetition = (const float *)ptr();
        if (rnd() % 2) a.n_bias = odd32(5), a.bias_id = (const int32_t *)ptr(), a.bias = (const float *)ptr();
        if (rnd() % 2) a.mask = (const uint32_t *)ptr(), a.mask_stride = odd64(4);
        st = dsim_logit_adjust(rnd() % 99 ? &a : nullptr, nullptr);
        st == DSIM_OK ? ++ok : ++refused;
    }
    printf("%ld calls accepted, %ld refused, %ld reached a launch\n", ok, refused, dsim::launches);
    return dsim::launches > 1000 && refused > 1000 ? 0 : 1;
}
