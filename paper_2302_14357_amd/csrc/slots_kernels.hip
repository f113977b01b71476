// Pages for prompts, and the places of a packed batch's tokens in them.
#include "op_device.h"

#define SLOTS_THREADS 256

// the sum over a workgroup's threads of smaller number, and (all) over all of them
__device__ __forceinline__ int64_t slots_before(int64_t x, int64_t *all) {
    __shared__ int64_t s_sum[SLOTS_THREADS / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t sum = x;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) {
        const int64_t y = __shfl_up(sum, i);
        if (lane >= i) sum += y;
    }
    __syncthreads();   // (the last call's sums have been read)
    if (lane == 63) s_sum[wave] = sum;
    __syncthreads();
    int64_t before = sum - x, total = 0;
#pragma unroll
    for (int i = 0; i < SLOTS_THREADS / 64; ++i) {
        before += i < wave ? s_sum[i] : 0;
        total += s_sum[i];
    }
    *all = total;
    return before;
}

struct TablesP {
    const int *lens, *free_pages, *taken;
    int *tables, *out_lens, *out_taken;
    int64_t ld;
    int prompts, beams, page, width, room, free_count, per;
};

struct TablesPrompt {
    int whole, own;   // pages that its rows share, and those that a row has for itself
    int64_t count;    // of all together (0: it takes none)
    bool live;
};

__device__ __forceinline__ TablesPrompt tables_prompt(const TablesP &p, int n) {
    TablesPrompt x = {0, 0, 0, false};
    if (n < 0) return x;
    const unsigned need = ((unsigned)n + (unsigned)p.room + (unsigned)p.page - 1) / (unsigned)p.page;   // (below 2^32: room is at most 2^30, page 2^16)
    if (need > (unsigned)p.width) return x;
    x.live = true;
    x.whole = (unsigned)n / (unsigned)p.page;
    x.own = (int)need - x.whole;
    x.count = x.whole + (int64_t)p.beams * x.own;
    return x;
}

#define TABLES_PER 64   // prompts of a workgroup at most

// One launch: a workgroup adds up the pages of all prompts before its own (the lengths come from the caches) and then writes its prompts' rows, a
// piece of a row by lanes side by side.  A prompt whose pages end behind the list's end has none, and so has every later one that wants any.
// 4096 prompts of up to 4000 tokens, four rows each of 257 columns: 11.5 us, 17 MB written (columns one after the other 12.9): behind the sums a thread has eight turns of loads and
// stores, of which each waits for the last one's.  Eight prompts 3.5: a call's latency.  65536 prompts of up to 40 tokens 55 us, 524288 1840: all lengths are added up in every workgroup.
// (A launch for the sums and one for the rows would be one latency more; adding up all lengths before its own costs a workgroup 16 loads a thread at most there.)
__global__ void __launch_bounds__(SLOTS_THREADS)
k_page_tables(TablesP p) {
    __shared__ int64_t s_base[TABLES_PER];
    __shared__ int s_whole[TABLES_PER], s_own[TABLES_PER];
    const int first = (int)blockIdx.x * p.per, mine = min(p.per, p.prompts - first), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t sum = 0, base;
    for (int i = threadIdx.x; i < first; i += 8 * SLOTS_THREADS) {
        int n[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            n[j] = -1;
            if (i + j * SLOTS_THREADS < first) n[j] = p.lens[i + j * SLOTS_THREADS];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += tables_prompt(p, n[j]).count;
    }
    slots_before(sum, &base);
    const int taken = max(*p.taken, 0);
    base += taken;
    if (p.prompts == 0 && threadIdx.x == 0) *p.out_taken = taken;
    if (wave == 0) {
        const int i = first + lane, n = lane < mine ? p.lens[i] : -1;
        const TablesPrompt x = tables_prompt(p, n);
        int64_t end = x.count;
#pragma unroll
        for (int j = 1; j < 64; j <<= 1) {
            const int64_t y = __shfl_up(end, j);
            if (lane >= j) end += y;
        }
        end += base;
        const bool fits = x.live && (x.count == 0 || end <= p.free_count);
        if (lane < mine) {
            s_base[lane] = end - x.count;
            s_whole[lane] = fits ? x.whole : 0;
            s_own[lane] = fits ? x.own : 0;
            for (int b = 0; b < p.beams; ++b) p.out_lens[(int64_t)i * p.beams + b] = fits && b == 0 ? n : -1;
            // the pages taken now: up to the end of the last prompt that is whole within the list
            if (end <= p.free_count && (i == p.prompts - 1 || end + tables_prompt(p, p.lens[i + 1]).count > p.free_count)) *p.out_taken = (int)end;
            if (i == 0 && end > p.free_count) *p.out_taken = taken;
        }
    }
    __syncthreads();
    // as many rows a wave at a time as fit into its lanes
    int cols = 1;
    while (cols < p.width && cols < 64) cols *= 2;
    const int step = SLOTS_THREADS / cols, rows = mine * p.beams;
    for (int r = threadIdx.x / cols; r < rows; r += step) {
        const int k = r / p.beams, whole = s_whole[k], own = s_own[k];
        const int *from = p.free_pages + s_base[k];
        const int64_t skip = (int64_t)(r - k * p.beams) * own;   // (the shared pages first, then those of its first row, its second ...)
        int *to = p.tables + ((int64_t)first * p.beams + r) * p.ld;
        for (int c = threadIdx.x & (cols - 1); c < p.width; c += 4 * cols) {
            int id[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int at = c + j * cols;
                id[j] = -1;
                if (at < whole + own) id[j] = from[at + (at < whole ? 0 : skip)];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j * cols < p.width) to[c + j * cols] = id[j];
        }
    }
}

struct SlotsP {
    const int *lens, *past, *tables;
    int *starts, *positions;
    int64_t *slots;
    int64_t ld;
    int prompts, tokens, width, page;
};

#define SLOTS_PER 4                                        // tokens a thread
#define SLOTS_TOKENS (SLOTS_THREADS * SLOTS_PER)
#define SLOTS_LENS (SLOTS_THREADS * 4)                     // lengths at a time

// One launch: a workgroup adds up the lengths until its tokens are reached, 1024 at a time, and looks each of its tokens up among the sums of the
// prompts that it can belong to; the last workgroup writes the sums themselves.
// A million tokens of 1000 prompts: 9.4 us, 12.6 MB written; of 40 prompts' 1200 tokens 5.0: the chain of lengths, sums, search and table.
__global__ void __launch_bounds__(SLOTS_THREADS)
k_page_slots(SlotsP p) {
    __shared__ int s_end[SLOTS_LENS];
    const bool writer = blockIdx.x == gridDim.x - 1;
    const int64_t t0 = (int64_t)blockIdx.x * SLOTS_TOKENS, t1 = min((int64_t)p.tokens, t0 + SLOTS_TOKENS);
    int prompt[SLOTS_PER], start[SLOTS_PER];
#pragma unroll
    for (int j = 0; j < SLOTS_PER; ++j) prompt[j] = -1, start[j] = 0;
    if (writer && threadIdx.x == 0) p.starts[0] = 0;
    int64_t carry = 0;
    for (int c0 = 0; c0 < p.prompts; c0 += SLOTS_LENS) {
        int64_t n[4], sum = 0, all;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = c0 + (int)threadIdx.x * 4 + j;
            n[j] = i < p.prompts ? max(p.lens[i], 0) : 0;
            sum += n[j];
        }
        int64_t end = carry + slots_before(sum, &all);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            end += n[j];
            const int e = (int)min(end, (int64_t)p.tokens);
            s_end[threadIdx.x * 4 + j] = e;
            if (writer && c0 + (int)threadIdx.x * 4 + j < p.prompts) p.starts[c0 + threadIdx.x * 4 + j + 1] = e;
        }
        __syncthreads();
        const int64_t next = carry + all;
        if (!writer && next > t0) {
#pragma unroll
            for (int j = 0; j < SLOTS_PER; ++j) {
                const int64_t t = t0 + threadIdx.x + j * SLOTS_THREADS;
                if (t >= t1 || t < carry || t >= next) continue;
                int low = 0;   // the first end above t
#pragma unroll
                for (int w = SLOTS_LENS / 2; w > 0; w /= 2)
                    if (s_end[low + w - 1] <= t) low += w;
                prompt[j] = c0 + low;
                start[j] = low > 0 ? s_end[low - 1] : (int)carry;
            }
        }
        carry = next;
        if (!writer && carry >= t1) break;
        __syncthreads();
    }
    if (writer) return;
#pragma unroll
    for (int j = 0; j < SLOTS_PER; ++j) {
        const int64_t t = t0 + threadIdx.x + j * SLOTS_THREADS;
        if (t >= t1) continue;
        int64_t at = -1, slot = -1;
        if (prompt[j] >= 0) {
            at = t - start[j] + (p.past ? max(p.past[prompt[j]], 0) : 0);
            const int64_t column = (unsigned)at / (unsigned)p.page;   // (below 2^32)
            if (column < p.width) {
                const int id = p.tables[prompt[j] * p.ld + column];
                if (id >= 0) slot = (int64_t)id * p.page + (at - column * p.page);
            }
        }
        p.positions[t] = (int)min(at, (int64_t)INT32_MAX);
        p.slots[t] = slot;
    }
}

extern "C" int tbs_page_tables(const tbs_page_tables_args *args, void *stream) {
    if (!args) return TBS_EINVAL;
    const tbs_page_tables_args &a = *args;
    if (a.prompts < 0 || a.beams < 1 || a.beams > 65535 || a.page < 1 || a.page > 65536 || a.table_width < 1 || a.room < 0 || a.room > (1 << 30) || a.free_count < 0 ||
        (int64_t)a.table_width * a.page > (1 << 30) || (int64_t)a.prompts * a.beams > INT32_MAX)
        return TBS_EINVAL;
    if (!a.taken || !a.out_taken) return TBS_EINVAL;
    if (a.prompts > 0 && (!a.lens || (!a.free_pages && a.free_count > 0) || !a.tables || !a.out_lens || a.ld_tables < a.table_width)) return TBS_EINVAL;
    // (a workgroup reads the lengths of others' prompts, and the whole list may be its own)
    const int64_t rows = (int64_t)a.prompts * a.beams;
    if (op_written_over({op_rows(a.tables, rows, a.ld_tables, a.table_width, 4), op_rows(a.out_lens, 1, rows, rows, 4), op_rows(a.out_taken, 1, 1, 1, 4)},
                        {op_rows(a.lens, 1, a.prompts, a.prompts, 4), op_rows(a.free_pages, 1, a.free_count, a.free_count, 4), op_rows(a.taken, 1, 1, 1, 4)}))
        return TBS_EINVAL;
    const hipStream_t st = (hipStream_t)stream;
    TablesP p = {a.lens, a.free_pages, a.taken, a.tables, a.out_lens, a.out_taken, a.ld_tables, a.prompts, a.beams, a.page, a.table_width, a.room, a.free_count, 1};
    p.per = a.prompts / 1024 < 1 ? 1 : a.prompts / 1024 < TABLES_PER ? a.prompts / 1024 : TABLES_PER;
    const int blocks = a.prompts / p.per + (a.prompts % p.per != 0);
    hipLaunchKernelGGL(k_page_tables, dim3(blocks > 0 ? blocks : 1), dim3(SLOTS_THREADS), 0, st, p);
    return hipGetLastError() == hipSuccess ? TBS_OK : TBS_EHIP;
}

extern "C" int tbs_page_slots(const tbs_page_slots_args *args, void *stream) {
    if (!args) return TBS_EINVAL;
    const tbs_page_slots_args &a = *args;
    if (a.prompts < 0 || a.tokens < 0 || a.page < 1 || a.page > 65536 || a.table_width < 1 || (int64_t)a.table_width * a.page > (1 << 30)) return TBS_EINVAL;
    if (!a.starts || (a.prompts > 0 && (!a.lens || !a.tables || a.ld_tables < a.table_width)) || (a.tokens > 0 && (!a.positions || !a.slots))) return TBS_EINVAL;
    // (every workgroup reads the lengths)
    if (op_written_over({op_rows(a.starts, 1, (int64_t)a.prompts + 1, (int64_t)a.prompts + 1, 4), op_rows(a.positions, 1, a.tokens, a.tokens, 4), op_rows(a.slots, 1, a.tokens, a.tokens, 8)},
                        {op_rows(a.lens, 1, a.prompts, a.prompts, 4), op_rows(a.past, 1, a.prompts, a.prompts, 4), op_rows(a.tables, a.prompts, a.ld_tables, a.table_width, 4)}))
        return TBS_EINVAL;
    const SlotsP p = {a.lens, a.past, a.tables, a.starts, a.positions, a.slots, a.ld_tables, a.prompts, a.tokens, a.table_width, a.page};
    const unsigned blocks = (unsigned)((a.tokens + (int64_t)SLOTS_TOKENS - 1) / SLOTS_TOKENS) + 1;
    hipLaunchKernelGGL(k_page_slots, dim3(blocks), dim3(SLOTS_THREADS), 0, (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? TBS_OK : TBS_EHIP;
}
