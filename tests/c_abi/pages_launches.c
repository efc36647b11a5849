/*
 * What the calls on pages and the differential attention launch, and what they say
 * when a launch fails.  Needs no GPU (hip_stub.h).  Test infrastructure only.
 */
#include "hip_stub.h"

#include "agft_diff.h"
#include "agft_pages.h"

static int failures;
#define CHECK(x) do { if (!(x)) { ++failures; printf("line %d: %s\n", __LINE__, #x); } } while (0)

/* device addresses: never read or written here */
static void *const A = (void *)0x10000000000ull, *const B = (void *)0x20000000000ull, *const C = (void *)0x30000000000ull,
            *const W = (void *)0x40000000000ull;
static int32_t *const I = (int32_t *)0x50000000000ull;
static const size_t BIG = (size_t)1 << 40;

int main(void)
{
    const agft_kv_config c = {64, 100, 1000, 32, 4, 8, 128, AGFT_KV_E4M3};

    /* forks: one launch up to 1,024, of at most 512 workgroups; two beyond, the second only after the first */
    for (int n = 1; n <= 65536; n = n < 1024 ? 1024 : n == 1024 ? 1025 : n * 8 - 1 < 65536 ? n * 8 - 1 : n < 65536 ? 65536 : 65537) {
        agft_kv_config t = c;
        t.requests = 65536;
        for (int rows = 1000; rows <= 3000; rows += 1000) {
            const int parts = (rows + 1023) / 1024;
            t.row_pages = rows;
            start(0);
            CHECK(agft_pages_fork(&t, A, BIG, I, I, NULL, n, C, BIG, n, NULL) == AGFT_OK);
            CHECK(n_ran == (n <= 1024 ? 1 : 2));
            const unsigned most = n <= 1024 ? 512 : 8192, all = (unsigned)n * parts;
            CHECK(ran_block[n_ran - 1] == 256 && ran_grid[n_ran - 1] == (all < most ? all : most));
            if (n > 1024) CHECK(ran_block[0] == 1024 && ran_grid[0] == 1);
            for (int fail = 1; fail <= (n <= 1024 ? 1 : 2); ++fail) {
                start(fail);
                CHECK(agft_pages_fork(&t, A, BIG, I, I, I, n, C, BIG, n, NULL) == AGFT_E_HIP && n_ran == fail - 1);
            }
        }
    }

    /* trims: three launches, requests in at most 1,024 chunks of at most 64 */
    for (int requests = 1; requests <= 65536; requests = requests < 64 ? requests * 8 : requests * 4) {
        agft_kv_config t = c;
        t.requests = requests;
        const unsigned per = (requests + 1023) / 1024, chunks = (requests + per - 1) / per;
        start(0);
        CHECK(agft_pages_trim(&t, A, BIG, I, C, BIG, 1, NULL) == AGFT_OK && n_ran == 3);
        for (int k = 0; k < 3; ++k) CHECK(ran_block[k] == 256 && ran_grid[k] == chunks);
        for (int fail = 1; fail <= 3; ++fail) {
            start(fail);
            CHECK(agft_pages_trim(&t, A, BIG, I, C, BIG, 1, NULL) == AGFT_E_HIP && n_ran == fail - 1);
        }
        start(0);
        CHECK(agft_pages_commit(&t, A, BIG, C, BIG, 1, NULL) == AGFT_OK && n_ran == 1 && ran_grid[0] == chunks);
        start(1);
        CHECK(agft_pages_commit(&t, A, BIG, C, BIG, 1, NULL) == AGFT_E_HIP);
    }

    /* compaction: one launch up to 2^18 pages, four beyond, of 32,768 pages a workgroup */
    const int pools[] = {1, 4096, 4097, 1 << 18, (1 << 18) + 1, 1 << 28};
    for (int k = 0; k < 6; ++k) {
        agft_kv_config t = c;
        t.pages = pools[k];
        const int moves = pools[k] < 2 ? 1 : pools[k] / 2, launches = pools[k] <= 1 << 18 ? 1 : 4;
        start(0);
        CHECK(agft_pages_compact(&t, A, BIG, C, BIG, moves, NULL) == AGFT_OK && n_ran == launches);
        if (launches == 1) CHECK(ran_block[0] == 1024 && ran_grid[0] == (unsigned)(pools[k] + 4095) / 4096);
        else for (int z = 0; z < 4; ++z) CHECK(z == 1 ? ran_grid[z] == 2048 : ran_grid[z] == (unsigned)((pools[k] + 32767) / 32768));
        for (int fail = 1; fail <= launches; ++fail) {
            start(fail);
            CHECK(agft_pages_compact(&t, A, BIG, C, BIG, moves, NULL) == AGFT_E_HIP && n_ran == fail - 1);
        }
        if (pools[k] > 3) {
            start(0);
            CHECK(agft_pages_compact(&t, A, BIG, C, BIG, moves - 1, NULL) == AGFT_E_INVAL && n_ran == 0);
        }
    }

    /* copies: 16 KB of a page a workgroup */
    for (int page = 16; page <= 128; page *= 2)
        for (int moves = 1; moves <= 100000; moves *= 10) {
            agft_kv_config t = c;
            t.page = page;
            const int parts = (4 * 2 * page * 128 + 16383) / 16384;
            start(0);
            CHECK(agft_pages_copy(&t, B, BIG, C, BIG, moves, NULL) == AGFT_OK && n_ran == 1 && ran_block[0] == 256);
            CHECK(ran_grid[0] == (unsigned)(moves * parts < 16384 ? moves * parts : 16384));
        }
    start(1);
    CHECK(agft_pages_copy(&c, B, BIG, C, BIG, 5, NULL) == AGFT_E_HIP);

    /* differential attention: requests of at most 16 query rows in one launch; many rows in a second one,
       of 64 numbers in the same where a request may have more than 64 */
    const agft_kv_dense q = {(void *)0x500000, 8192, 128, AGFT_KV_BF16};
    const agft_diff_args d = {(const float *)I, 0, 1, NULL, 1e-5f, 1.0f};
    for (int dim = 64; dim <= 128; dim *= 2) {
        agft_kv_config t = c;
        t.dim = dim;
        const agft_kv_dense out = {(void *)0x600000, 8192, 2 * dim, AGFT_KV_BF16};
        const unsigned groups = dim == 64 ? 768 : 512;
        /* 200 x 8 rows: 12 tiles of 128, one more for each of 64 requests, 512 / 4 shared ones; 2 pairs */
        const unsigned tiles = (12 + 64 + 128) * 2 * (dim == 64 ? 2 : 1);
        for (int max_new = 1; max_new <= 20; ++max_new) {
            const int beside = dim == 64 && max_new > 8, launches = max_new <= 2 || beside ? 1 : 2;
            start(0);
            CHECK(agft_diff_attend(&t, A, BIG, B, BIG, C, BIG, 200, max_new, &q, &d, &out, NULL, 0.1f, W, BIG, NULL) == AGFT_OK);
            CHECK(n_ran == launches);
            if (!beside) CHECK(ran_block[0] == 256 && ran_grid[0] == groups);
            if (max_new > 2) CHECK(ran_block[launches - 1] == (dim == 64 ? 256u : 512u) && ran_grid[launches - 1] == tiles + (beside ? groups : 0));
            for (int fail = 1; fail <= launches; ++fail) {
                start(fail);
                CHECK(agft_diff_attend(&t, A, BIG, B, BIG, C, BIG, 200, max_new, &q, &d, &out, NULL, 0.1f, W, BIG, NULL) == AGFT_E_HIP);
                CHECK(n_ran == fail - 1);
            }
        }
    }

    printf("%d failures\n", failures);
    return failures != 0;
}
