/*
 * Calls the cache's entry points over valid, extreme and invalid arguments,
 * none of which enqueues work; built with the host sanitizers.  Test
 * infrastructure only.
 */
#include <limits.h>
#include <stdio.h>

#include "agft_kv.h"

static int failures;
#define CHECK(x) do { if (!(x)) { ++failures; printf("line %d: %s\n", __LINE__, #x); } } while (0)

int main(void)
{
    static const int32_t odd[] = {INT_MIN, -1, 0, 1, 2, 15, 16, 17, 64, 128, 256, 257, 65536, 1 << 26, 1 << 28, INT_MAX};
    enum { N = sizeof(odd) / sizeof(odd[0]) };
    void *p = (void *)0x100000;
    const agft_kv_config good = {65536, (1 << 30) / 128 - 1, 1 << 28, 128, 256, 128, 256, AGFT_KV_INT8};
    agft_kv_dense d = {p, 1 << 20, 256, AGFT_KV_BF16}, none = {0};
    CHECK(agft_kv_cache_bytes(&good) > (size_t)1 << 52 && agft_kv_tables_bytes(&good) > (size_t)1 << 41);
    CHECK(agft_kv_step_bytes(&good, 1 << 30) > (size_t)1 << 33 && agft_kv_attend_bytes(&good, 1 << 30) > 0);
    for (int f = 0; f < 8; ++f)
        for (int i = 0; i < N; ++i) {
            agft_kv_config c = good;
            ((int32_t *)&c)[f] = odd[i];
            agft_kv_tables_view tv;
            agft_kv_step_view sv;
            const size_t t = agft_kv_tables_bytes(&c), k = agft_kv_cache_bytes(&c);
            CHECK((t == 0) == (k == 0));
            CHECK((agft_kv_tables_at(&c, p, SIZE_MAX, &tv) == AGFT_OK) == (t != 0));
            for (int j = 0; j < N; ++j) {
                const size_t s = agft_kv_step_bytes(&c, odd[j]), a = agft_kv_attend_bytes(&c, odd[j]);
                CHECK((s == 0) == (a == 0) && (t != 0 || s == 0));
                CHECK((agft_kv_step_at(&c, odd[j], p, SIZE_MAX, &sv) == AGFT_OK) == (s != 0));
                CHECK(agft_kv_plan(&c, p, SIZE_MAX, NULL, p, SIZE_MAX, odd[j], NULL) < 0);
                CHECK(agft_kv_append(&c, p, SIZE_MAX, p, SIZE_MAX, odd[j], &d, &none, NULL) < 0);
                CHECK(agft_kv_attend(&c, p, SIZE_MAX, p, SIZE_MAX, p, SIZE_MAX, odd[j], 1, &none, &d, NULL, 1.0f, p, SIZE_MAX,
                                     NULL) < 0);
                CHECK(agft_kv_commit(&c, p, 0, p, SIZE_MAX, odd[j], NULL) < 0);
            }
            CHECK(agft_kv_export(&c, p, SIZE_MAX, (int64_t *)p, INT64_MAX, &d, &d, NULL) < 0);
            CHECK(agft_kv_reset(&c, NULL, SIZE_MAX, NULL) < 0);
        }
    printf("%d failures\n", failures);
    return failures != 0;
}
