/*
 * What the cache's calls launch, and what they say when a launch fails.  Needs
 * no GPU (hip_stub.h).  Test infrastructure only.
 */
#include "hip_stub.h"

#include "agft_kv.h"

static int failures;
#define CHECK(x) do { if (!(x)) { ++failures; printf("line %d: %s\n", __LINE__, #x); } } while (0)

/* device addresses: never read or written here */
static void *const A = (void *)0x10000000000ull, *const B = (void *)0x20000000000ull, *const C = (void *)0x30000000000ull,
            *const W = (void *)0x40000000000ull;
static const size_t BIG = (size_t)1 << 40;

int main(void)
{
    agft_kv_config c = {64, 100, 1000, 32, 4, 8, 128, AGFT_KV_E4M3};
    agft_kv_dense d = {(void *)0x500000, 8192, 128, AGFT_KV_BF16};

    /* tables: one launch up to 1,024 requests, two beyond, the second only after the first */
    for (int requests = 1023; requests <= 1026; ++requests) {
        agft_kv_config t = c;
        t.requests = requests;
        start(0);
        CHECK(agft_kv_plan(&t, A, BIG, B, C, BIG, 5000, NULL) == AGFT_OK);
        CHECK(n_ran == (requests <= 1024 ? 1 : 2));
        CHECK(ran_block[n_ran - 1] == 256 && ran_grid[n_ran - 1] == 20);
        if (requests > 1024) CHECK(ran_block[0] == 1024 && ran_grid[0] == 2);
        start(1);
        CHECK(agft_kv_plan(&t, A, BIG, B, C, BIG, 5000, NULL) == AGFT_E_HIP && n_ran == 0);
    }
    {
        agft_kv_config t = c;
        t.requests = 2000;
        start(2);
        CHECK(agft_kv_plan(&t, A, BIG, B, C, BIG, 5000, NULL) == AGFT_E_HIP && n_ran == 1);
    }
    start(0);
    CHECK(agft_kv_plan(&c, A, BIG, B, C, BIG, 1 << 30, NULL) == AGFT_OK && ran_grid[0] == 512);
    start(0);
    CHECK(agft_kv_reset(&c, A, BIG, NULL) == AGFT_OK && agft_kv_commit(&c, A, BIG, C, BIG, 9, NULL) == AGFT_OK && n_ran == 2);

    /* writes: a workgroup per run at most, 16 tokens of a page per wavefront */
    for (int page = 16; page <= 128; page *= 2)
        for (int tokens = 1; tokens <= 3000; tokens += 733) {
            agft_kv_config t = c;
            t.page = page;
            const int runs = 2 * t.requests + tokens / page < tokens ? 2 * t.requests + tokens / page : tokens;
            start(0);
            CHECK(agft_kv_append(&t, A, BIG, C, BIG, tokens, &d, &d, NULL) == AGFT_OK);
            CHECK(n_ran == 1 && ran_block[0] == 4u * page && ran_grid[0] == (unsigned)runs);
        }
    start(1);
    CHECK(agft_kv_append(&c, A, BIG, C, BIG, 5, &d, &d, NULL) == AGFT_E_HIP);

    /* exports: 64 slots per workgroup, none for none */
    for (int n = 0; n <= 200; ++n) {
        start(0);
        CHECK(agft_kv_export(&c, A, BIG, B, n, &d, &d, NULL) == AGFT_OK);
        CHECK(n ? n_ran == 1 && ran_grid[0] == (unsigned)(n + 63) / 64 : n_ran == 0);
    }

    /* attention: requests of at most 16 query rows in one launch, a second one
       where a request may have up to 64, both kinds in one where it may have more */
    for (int dim = 64; dim <= 256; dim *= 2) {
        const void *few = NULL, *many = NULL;
        for (int max_new = 1; max_new <= 20; ++max_new) {
            agft_kv_config t = c;
            t.dim = dim;
            const unsigned groups = dim == 64 ? 1024 : dim == 128 ? 768 : 512;
            /* 200 x 8 rows: 12 tiles of 128, one more for each of 64 requests, 512 / 4 shared ones; 4 heads */
            const unsigned tiles = (12 + 64 + 128) * 4;
            start(0);
            CHECK(agft_kv_attend(&t, A, BIG, B, BIG, C, BIG, 200, max_new, &d, &d, NULL, 0.1f, W, BIG, NULL) == AGFT_OK);
            CHECK(n_ran == (max_new > 2 && max_new <= 8 ? 2 : 1) && ran_block[0] == 256 && ran_block[n_ran - 1] == 256);
            if (max_new == 1) few = ran[0];
            if (max_new == 3) many = ran[1];
            if (max_new <= 8) CHECK(ran[0] == few && ran_grid[0] == groups);
            if (max_new > 2) CHECK(ran[n_ran - 1] == many && ran_grid[n_ran - 1] == tiles + (max_new > 8 ? groups : 0));
        }
        CHECK(few != many);
    }
    for (int fail = 1; fail <= 2; ++fail) {
        start(fail);
        CHECK(agft_kv_attend(&c, A, BIG, B, BIG, C, BIG, 200, 5, &d, &d, NULL, 0.1f, W, BIG, NULL) == AGFT_E_HIP);
        CHECK(n_ran == fail - 1);
    }

    printf("%d failures\n", failures);
    return failures != 0;
}
