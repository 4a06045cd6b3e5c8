// Runs workgroups of preft_kv_plan's launch on the CPU (tests/test_kv_plan_host.py).  All tables but the block table are heap blocks of exactly their size, so that with a
// sanitizer an access past one ends the run.  Standard input: S T MAX_PAGES N_FREE PAGE BLOCK, then REPEAT, that many times LO HI for the offsets, one more offset each for the rest up to S + 1, and CTX for all
// requests.  BLOCK: the workgroup to run, from the end if negative; -1000000: all.  Prints counts and the sums of positions and slots that were written.
// With an argument: rows T of a store each, and prints what preft_kv_store returns and the workgroups that it launches.
#include "emulated_hip.hpp"

#include <sys/mman.h>

constexpr long long NO_BLOCK = -(1ll << 40);
static long long which_block;
static unsigned launched_grid;
template <typename K, typename A> void emulated_launch(K kernel, dim3 grid, dim3 threads, const A &args)
{
    launched_grid = grid.x;
    if (which_block == NO_BLOCK) return;
    for (unsigned b = 0; b < grid.x; ++b) {
        const long long from_end = (long long)b - grid.x;
        if (which_block == -1000000 || which_block == (long long)b || which_block == from_end) emulated::run_block(threads.x, b, grid.x, [&] { kernel(args); });
    }
}
#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(kernel, grid, threads, lds, stream, args) emulated_launch(kernel, grid, threads, args)
#define hipGetLastError() hipSuccess

#include "../paper_2605_14217_amd/csrc/kv_pages.hip"

// workgroups that preft_kv_store launches for T rows; none is run, and no pointer is followed
static int ask_store(long long T)
{
    char *const at = reinterpret_cast<char *>(1ull << 44);
    which_block = NO_BLOCK;
    return preft_kv_store(at, at + (1ll << 30), 4, 16, at + (1ll << 40), 64, at + (1ll << 41), 64, (int32_t)T, 1, 64, reinterpret_cast<const int64_t *>(at), PREFT_BF16, nullptr);
}

int main(int argc, char **)
{
    long long S, T, max_pages, n_free, page, repeat;
    if (argc > 1) {                                    // rows of stores
        while (std::scanf("%lld", &T) == 1) {
            const int rc = ask_store(T);
            std::printf("%d %u\n", rc, launched_grid);
        }
        return 0;
    }
    while (std::scanf("%lld %lld %lld %lld %lld %lld %lld", &S, &T, &max_pages, &n_free, &page, &which_block, &repeat) == 7) {
        std::vector<int32_t> start;
        long long lo, hi, ctx, v;
        if (std::scanf("%lld %lld", &lo, &hi) != 2) return 2;
        for (long long i = 0; i < repeat; ++i) { start.push_back((int32_t)lo); start.push_back((int32_t)hi); }
        while ((long long)start.size() < S + 1) {
            if (std::scanf("%lld", &v) != 1) return 2;
            start.push_back((int32_t)v);
        }
        if (std::scanf("%lld", &ctx) != 1) return 2;
        // the block table may be larger than memory: pages that nobody touches take none
        const size_t table_bytes = (size_t)S * max_pages * 4 + 4096;
        int32_t *table = (int32_t *)mmap(nullptr, table_bytes, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0);
        if (table == MAP_FAILED) return 4;
        std::vector<int32_t> at(T, -7), kv(S, -7), counts(2, -7), ctx_len(S, (int32_t)ctx), free_pages(n_free);
        std::vector<int64_t> slot(T, -7);
        for (long long i = 0; i < n_free; ++i) free_pages[i] = (int32_t)i;
        const int rc = preft_kv_plan(slot.data(), at.data(), kv.data(), table, max_pages, (int32_t)max_pages, counts.data(), start.data(), ctx_len.data(), (int32_t)S, (int32_t)T,
                                     free_pages.data(), (int32_t)n_free, (int32_t)page, nullptr);
        munmap(table, table_bytes);
        long long sum_at = 0, sum_slot = 0, rows = 0;
        for (long long t = 0; t < T; ++t)
            if (at[t] != -7) { ++rows; sum_at += at[t]; sum_slot += slot[t]; }
        std::printf("%d %u %d %d %lld %lld %lld\n", rc, launched_grid, counts[0], counts[1], rows, sum_at, sum_slot);
        std::fflush(stdout);
    }
    return 0;
}
