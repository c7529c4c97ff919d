// Page tables, packed offsets, positions and slots of a step from the requests' lengths (include/emm_step.h has the rules).
//
// Every request gives pages back or takes some, which page that is follows from how many those before it gave and took: three
// running sums over the requests (pages given back, pages taken, tokens), and then every page moved and every token by itself.
// The stack of free pages is never walked.  Let c pages lie on it and the requests give back R, in order; then page i of the
// stack is free_pages[i] for i < c and the (i - c)-th given back for c <= i < c + R, which a search in the running sums finds in
// its request's table; and the j-th page taken is page c + R - 1 - j.  So a workgroup needs nothing of another: each takes the sums
// by itself (they are of a few numbers per request) and its share of the pages and tokens, and writes nothing that another reads, but
// where an output is the input that it follows: then a second, small launch writes those, or one workgroup does it all.
//
// Bound by the chain of its round trips: arguments, lengths, page ids, stores.  In a graph, us: 64 requests' decode step behind a window 3.7 (5.1 with the
// three kinds of work one after the other and two running sums in every call; without a window 3.1), 32000 tokens of 48 prompts 4.2, in place 6.3; an empty kernel is 1.7.
#include "step_internal.h"

namespace emm {

namespace {

constexpr int SAT = MOST_STEP_PAGES;                     // sums stop here: whatever the arrays hold, nothing wraps

__device__ inline int sat_add(int x, int y) { return min((int)((unsigned)x + (unsigned)y), SAT); }       // 0 .. SAT each

// running sums over the wave's lanes, inclusive
__device__ inline int scan_wave(int x)
{
    x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true));      // row_shr:1, 2, 4, 8
    x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true));
    x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true));
    x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true));
    x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));     // row 0's sum to row 1, row 2's to row 3,
    x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));     // and row 1's to rows 2 and 3
    return x;
}

// Running sums of N numbers per thread over the workgroup, inclusive; `total` of all.  `part`: [N][waves] of LDS that nobody else uses.
template <int N, int NT>
__device__ inline void scan_block(int (&x)[N], int (&total)[N], int (*part)[NT / 64])
{
    constexpr int WAVES = NT / 64;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        x[n] = scan_wave(x[n]);
        if (lane == 63) part[n][wave] = x[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
        int before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const int p = part[n][w];
            all = sat_add(all, p);
            if (w < wave) before = sat_add(before, p);
        }
        x[n] = sat_add(x[n], before);
        total[n] = all;
    }
}

enum Mode { ALL, NO_STATE /* all but the outputs that may be inputs */, STATE /* those alone */ };

// ITEMS neighbouring requests per thread: up to NT * ITEMS
template <int NT, int ITEMS, int MODE>
__global__ __launch_bounds__(NT) void page_step_kernel(PageStepArgs a)
{
    constexpr int REQS = NT * ITEMS;
    __shared__ int back_end[REQS], first_back[REQS], need_end[REQS], cu_end[REQS], len_of[REQS];
    __shared__ int part[3][NT / 64], part2[2][NT / 64], odd[NT / 64];
    const int tid = threadIdx.x;
    const int ps_log2 = 4 + a.page_shift, ps = 1 << ps_log2, width = a.max_pages, n = a.num_reqs;
    const int row_slots = (int)min((long long)width << ps_log2, 1ll << 30);

    // ---- what each request gives back and needs
    int len[ITEMS], add[ITEMS], held[ITEMS], back[ITEMS], need[ITEMS], start[ITEMS];
    bool fits[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int r = tid * ITEMS + i;
        const bool here = r < n;
        len[i] = here ? a.lens[r] : 0;
        add[i] = here ? a.add_lens[r] : 0;
        held[i] = here ? a.held_from[r] : 0;
    }
    const int count = min(max(a.free_count[0], 0), a.num_pages);
    int sums[3] = {0, 0, 0};                                 // of back, need and tokens, of this thread's requests
    bool misfit = false;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const bool here = tid * ITEMS + i < n;
        len[i] = min(max(len[i], 0), row_slots);
        add[i] = max(add[i], 0);
        start[i] = max(held[i], a.sink_pages);
        held[i] = start[i];
        if (a.window > 0 && here) held[i] = max(start[i], max(len[i] - a.window + 1, 0) >> ps_log2);
        back[i] = held[i] - start[i];
        fits[i] = add[i] <= row_slots - len[i];
        if (!fits[i]) add[i] = -1;                           // (refused whatever is free)
        misfit = misfit || !fits[i];
        const int m = max(add[i], 0);
        need[i] = ((len[i] + m + ps - 1) >> ps_log2) - ((len[i] + ps - 1) >> ps_log2);
        sums[0] = sat_add(sums[0], back[i]);
        sums[1] = sat_add(sums[1], need[i]);
        sums[2] = sat_add(sums[2], m);
    }
    int total[3], mine[3] = {sums[0], sums[1], sums[2]};
    __shared__ int taken_s;
    if (tid == 0) taken_s = 0;
    if (__builtin_amdgcn_ballot_w64(misfit) != 0) odd[tid >> 6] = 1;
    else odd[tid >> 6] = 0;
    scan_block<3, NT>(sums, total, part);                    // (its barrier is the one behind which the others see these)
#pragma unroll
    for (int k = 0; k < NT / 64; ++k) misfit = misfit || odd[k] != 0;
    const int free_now = sat_add(count, total[0]);           // pages on the stack before any is taken

    // ---- who is served, and the packed offsets.  Of those that need pages the served ones are the first: the sum of all up to and
    //      with them is what the stack holds.
    // Mostly everybody is, and the offsets are the sums that there are; else they are taken again.
    const bool all_served = !misfit && total[1] <= free_now;
    int new_len[ITEMS], ends[2] = {0, 0};                    // tokens; requests refused
    int need_at[ITEMS], back_at[ITEMS];
    {
        int at_back = sums[0] - mine[0], at_need = sums[1] - mine[1];
        if (sums[0] >= SAT || sums[1] >= SAT) at_back = at_need = SAT;       // (beyond any pool: of no meaning)
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            at_back = sat_add(at_back, back[i]);
            at_need = sat_add(at_need, need[i]);
            back_at[i] = at_back;
            need_at[i] = at_need;
            const bool served = fits[i] && (need[i] == 0 || at_need <= free_now);
            new_len[i] = served ? add[i] : 0;
            if (!served) need[i] = 0;
            ends[0] = sat_add(ends[0], new_len[i]);
            if (!served && add[i] != 0 && tid * ITEMS + i < n) ends[1] += 1;
        }
    }
    int total2[2] = {total[2], 0}, mine_new = ends[0], taken = total[1];
    if (all_served) {
        ends[0] = sums[2];
    } else {
        // pages taken: the running sum at the last served request that needs some
        int taken_here = 0;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (need[i] > 0) taken_here = need_at[i];
        scan_block<2, NT>(ends, total2, part2);
        if (taken_here > 0) atomicMax(&taken_s, taken_here); // (a maximum of whole numbers: the same in any order)
    }
    {
        int at = ends[0] - mine_new;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int r = tid * ITEMS + i;
            at = sat_add(at, new_len[i]);
            if (r < n) {
                back_end[r] = back_at[i];
                first_back[r] = start[i] - (back_at[i] - back[i]);           // entry of the n-th page given back: first_back + n
                need_end[r] = need_at[i];
                cu_end[r] = at;
                len_of[r] = len[i];
                if (blockIdx.x == 0) {
                    if (MODE != STATE) {
                        a.prefix_lens[r] = len[i];
                        a.new_lens[r] = new_len[i];
                        a.cu_new_lens[r + 1] = at;
                    }
                    if (MODE != NO_STATE) {
                        a.lens_out[r] = len[i] + new_len[i];
                        a.held_out[r] = held[i];
                    }
                }
            }
        }
    }
    __syncthreads();
    if (!all_served) taken = taken_s;
    const int tokens = min(total2[0], a.max_tokens), left = free_now - taken;
    if (blockIdx.x == 0 && tid == 0) {
        if (MODE != NO_STATE) a.free_count_out[0] = min(left, a.num_pages);
        if (MODE != STATE) {
            a.cu_new_lens[0] = 0;
            if (a.refused != nullptr) a.refused[0] = total2[1];
        }
    }
    if (MODE == STATE) return;

    auto first_beyond = [&](const int* end, int x) -> int {  // the first request whose running sum is beyond x
        int lo = 0, hi = n;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (end[mid] > x) hi = mid; else lo = mid + 1;
        }
        return min(lo, n - 1);
    };
    auto given_back = [&](int nth) -> const int32_t* {       // where the n-th page given back stands
        const int r = first_beyond(back_end, nth);
        return a.page_table + (long long)r * width + min(max(first_back[r] + nth, 0), width - 1);
    };
    auto page_taken = [&](int j) -> int {                    // the j-th page taken
        const int i = free_now - 1 - j;
        if (i >= count) return *given_back(i - count);
        return a.free_pages[min(max(i, 0), a.num_pages - 1)];
    };
    const int stride = gridDim.x * NT;
    const int pushed = min(left, a.num_pages) - count;       // pages that were given back and not taken lie on the stack
    // Whole waves of each of the three kinds, one kind after the other, so that their chains of loads run side by side.
    auto waves = [](int n) { return (max(n, 0) + 63) & ~63; };
    const int first_pop = waves(pushed), first_token = first_pop + waves(taken), end = first_token + a.max_tokens;
    for (int item = blockIdx.x * NT + tid; item < end; item += stride) {
        if (item < first_pop) {
            if (item < pushed) a.free_pages[count + item] = *given_back(item);
        } else if (item < first_token) {
            const int x = item - first_pop;
            if (x >= taken) continue;
            const int r = first_beyond(need_end, x);
            const int before = r > 0 ? need_end[r - 1] : 0;
            const int entry = ((len_of[r] + ps - 1) >> ps_log2) + x - before;
            if (entry < width) a.page_table[(long long)r * width + entry] = page_taken(x);
        } else {
            const int x = item - first_token;
            int position = 0;
            int64_t slot = -1;
            if (x < tokens) {
                const int r = first_beyond(cu_end, x);
                position = len_of[r] + x - (r > 0 ? cu_end[r - 1] : 0);
                const int have = (len_of[r] + ps - 1) >> ps_log2, entry = position >> ps_log2;
                if (a.slots != nullptr) {
                    const int page = entry < have ? a.page_table[(long long)r * width + min(entry, width - 1)]
                                                  : page_taken((r > 0 ? need_end[r - 1] : 0) + entry - have);
                    slot = (int64_t)page * ps + (position & (ps - 1));
                }
            }
            if (a.positions != nullptr) a.positions[x] = position;
            if (a.slots != nullptr) a.slots[x] = slot;
        }
    }
}

template <int NT, int ITEMS>
hipError_t launch(const PageStepArgs& a, bool in_place, hipStream_t stream)
{
    // Where outputs are inputs one workgroup does it all up to so many tokens per thread, as the second launch costs 1.2 to 2.5 us; us of one workgroup and of
    // many with the second launch: 8 requests' 512 tokens 3.4 and 5.0, 1024 4.6 and 5.1, 2048 6.9 and 5.1.
    // Apart, many are never slower: 256 tokens 3.3 and 3.4, 1024 5.0 and 3.4, 8192 21.4 and 3.6.
    constexpr int ALONE = 4;
    constexpr int MOST_GROUPS = 256;
    const int groups = (int)min(((long long)a.max_tokens + NT - 1) / NT, (long long)MOST_GROUPS);
    if (groups <= (in_place ? ALONE : 1)) {
        hipLaunchKernelGGL((page_step_kernel<NT, ITEMS, ALL>), dim3(1), dim3(NT), 0, stream, a);
    } else if (!in_place) {
        hipLaunchKernelGGL((page_step_kernel<NT, ITEMS, ALL>), dim3(groups), dim3(NT), 0, stream, a);
    } else {
        hipLaunchKernelGGL((page_step_kernel<NT, ITEMS, NO_STATE>), dim3(groups), dim3(NT), 0, stream, a);
        hipLaunchKernelGGL((page_step_kernel<NT, ITEMS, STATE>), dim3(1), dim3(NT), 0, stream, a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_page_step(const PageStepArgs& a, bool in_place, hipStream_t stream)
{
    // Fewer waves meet sooner, and more requests a thread take longer; us of decode steps without a window, outputs apart from inputs: 64 requests with 256 threads 3.2, with 1024
    // 5.0; 300 with 256 x 4 requests 5.0, 512 x 2 4.7, 1024 x 1 5.5; 1000 5.9, 5.5, 7.1 (in place 11.4, 7.1, 6.7); 2000 with 1024 x 4 8.9, 512 x 8 11.3; 512
    // requests' 16384 tokens 5.2, 4.9, 6.6.
    if (a.num_reqs <= 256) return launch<256, 1>(a, in_place, stream);
    if (a.num_reqs <= 1024) return launch<512, 2>(a, in_place, stream);
    return launch<1024, MOST_STEP_REQS / 1024>(a, in_place, stream);
}

}  // namespace emm
