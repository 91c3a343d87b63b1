// Eviction: of every sequence that holds more than `budget` tokens the first and the most recent ones stay, and of those between
// them the ones with the largest mass (ties to the lower place); what stays moves together, in its order, in all pools.
//
// Three launches.  A workgroup per sequence finds the value at which its middle is cut (radix selection on the bits of the masses, three
// passes of 11, 11 and 10 bits), lists what stays, and says which of its pages change.  One workgroup looks up free pages for those of them
// that have another holder.  The last launch copies, and brings tables, lengths, holders and masses up to date.
// A kept token never moves up, and neither does one behind it move below: a workgroup that has a head's tokens of one plane, and reads some
// of them before it writes these, needs no second copy.  Pages are decided on as they were held when the call began, so that none
// that is given back is written while another sequence reads it.
// Bound by the copies: what is kept of the changed pages is read and written once.  32 sequences of up to 4500 tokens cut to 2048 in six pools
// (8 heads of 128, bf16; 1.6 GB read and written together) 354 us: selection 15, pages 5, copies 333 at 4.7 TB/s, where a large copy has 5.1.  24 of up
// to 160 cut to 128 in four pools (12 heads of 64, float32) 28 us: 10, 5 and 13, each a chain of few loads.  48 that share a prompt's pages cut to 600 79: 9, 6 and 64.
#include "page_lists.h"

namespace approxifer {

namespace {

// length: tokens before the call; low: first page that changes; need: pages that it wants, then where they begin in the list.
struct EvictPlan {
    int status, cut, length, low, need, offset;
};
// Workspace.  pages [B][after]: where the kept tokens go, page by page: a page, or -1 - n for the n-th that the sequence wants; sources [B][budget]:
// the pages that they come from; list [P]: free pages.
struct EvictSpace {
    EvictPlan *plans;
    int32_t *pages, *sources, *list;
};
struct EvictCall {
    int32_t *table, *lens, *refs;
    float *mass;
    int64_t mass_stride;
    int32_t *kept, *status;
    int B, M, P, shift, budget, first, recent;
    __device__ __host__ __forceinline__ int after() const { return static_cast<int>((budget + (int64_t{1} << shift) - 1) >> shift); }
    __device__ __forceinline__ int before(int length) const {
        return static_cast<int>((static_cast<int64_t>(length) + (1 << shift) - 1) >> shift);
    }
};

// Unsigned numbers in the order of the masses; both zeros are the same, NaN is below everything.
__device__ __forceinline__ unsigned ordered(float x) {
    const unsigned u = __float_as_uint(x + 0.0f);
    return x != x ? 0u : u >> 31 ? ~u : u | 0x80000000u;
}

constexpr int kBins = 2048;
constexpr int kEach = 4;                                      // places next to each other that a thread looks at

// A sequence that is cut: lists what stays of its middle, the places first..end-1, by kT threads; kHeld: there are no more of them than a
// thread can hold kEach of.  Returns the first place that moves.
template <int kT, bool kHeld>
__device__ __forceinline__ int select_kept(const EvictCall &c, const float *mass, const int32_t *row, int end, int32_t *kept, int32_t *sources,
                                           int *bins, int *sums, int *found) {
    const int thread = threadIdx.x, most = c.budget - c.first - c.recent;         // as many of them stay
    unsigned held[kEach];
    int pages[kEach];
    const auto look = [&](int j0) {                           // the keys of places j0.. (0 behind the end, as NaN: they are not counted)
        float x[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int j = min(j0 + k, end - 1);
            x[k] = mass[j];
            pages[k] = row[j >> c.shift];
        }
#pragma unroll
        for (int k = 0; k < kEach; ++k) held[k] = ordered(x[k]);
    };
    if (kHeld) look(c.first + kEach * thread);
    const auto keep = [&](int place, int page, int at) {
        kept[at] = place;
        sources[at] = page;
    };
    for (int j = thread; j < c.first; j += kT) keep(j, row[j >> c.shift], j);
    for (int n = thread; n < c.recent; n += kT) keep(end + n, row[(end + n) >> c.shift], c.budget - c.recent + n);
    if (thread == 0) found[2] = c.budget - c.recent;          // the first that moves: one of the middle, or the first recent one
    if (most == 0) {
        __syncthreads();
        return found[2];
    }
    unsigned cut = 0;                                         // the value of the last that stays; `rank` of those that have it do
    int rank = most;
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        for (int n = thread; n < kBins; n += kT) bins[n] = 0;
        __syncthreads();
        const auto count = [&](unsigned u) {
            if (pass == 0 || (u >> shift >> bits) == (cut >> shift >> bits)) atomicAdd(&bins[u >> shift & ((1 << bits) - 1)], 1);
        };
        if (kHeld) {
#pragma unroll
            for (int k = 0; k < kEach; ++k)
                if (c.first + kEach * thread + k < end) count(held[k]);
        } else {
            for (int j = c.first + thread; j < end; j += kT) count(ordered(mass[j]));
        }
        __syncthreads();
        constexpr int kOwn = kBins / kT;                      // bins of a thread, from the largest down
        int in[kOwn], mine = 0, total;
#pragma unroll
        for (int n = 0; n < kOwn; ++n) mine += in[n] = bins[kBins - 1 - kOwn * thread - n];
        int above = block_scan(mine, sums, &total);
#pragma unroll
        for (int n = 0; n < kOwn; ++n) {
            if (above < rank && rank <= above + in[n]) {
                found[0] = kBins - 1 - kOwn * thread - n;
                found[1] = rank - above;
            }
            above += in[n];
        }
        __syncthreads();
        cut |= static_cast<unsigned>(found[0]) << shift;
        rank = found[1];
    }
    int from = c.budget, larger = 0, equal = 0;               // of the stretches before this one
    for (int j0 = c.first; j0 < end; j0 += kEach * kT) {
        const int j = j0 + kEach * thread;
        if (!kHeld) look(j);
        int counts = 0;
#pragma unroll
        for (int k = 0; k < kEach; ++k)                       // at most 4096 of each
            if (j + k < end) counts += (held[k] > cut) + ((held[k] == cut) << 16);
        int total;
        const int before = block_scan(counts, sums, &total);
        int l = larger + (before & 0xffff), e = equal + (before >> 16);
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            if (j + k >= end) break;
            if (held[k] > cut || (held[k] == cut && e < rank)) {
                const int at = c.first + l + min(e, rank);
                keep(j + k, pages[k], at);
                if (at != j + k) from = min(from, at);
            }
            l += held[k] > cut;
            e += held[k] == cut;
        }
        larger += total & 0xffff;
        equal += total >> 16;
    }
    for (int o = 32; o > 0; o >>= 1) from = min(from, __shfl_xor(from, o));
    if (lane_id() == 0 && from < c.budget) atomicMin(&found[2], from);
    __syncthreads();
    return found[2];
}

// A workgroup per sequence.  What it waits for are the steps of three passes, each of which ends in a scan of the bins: 15 us for 4500 places,
// of which 1024 threads look at four each without asking for them again; 11 for 160 with 256 threads.
template <int kT>
__global__ __launch_bounds__(kT) void evict_select_kernel(EvictCall c, EvictSpace w) {
    __shared__ int bins[kBins];
    __shared__ int sums[16];
    __shared__ int found[3];
    const int b = blockIdx.x, thread = threadIdx.x, length = c.lens[b], mask = (1 << c.shift) - 1;
    int32_t *const kept = c.kept + static_cast<int64_t>(b) * c.budget, *const sources = w.sources + static_cast<int64_t>(b) * c.budget;
    const int32_t *const row = c.table + static_cast<int64_t>(b) * c.M;
    EvictPlan plan{APPROXIFER_GROUP_OK, 0, length, 0, 0, 0};
    bool bad = false;                                         // a page that nobody holds could be given to somebody else meanwhile
    if (length < 0 || length > (static_cast<int64_t>(c.M) << c.shift) || length > c.mass_stride) {
        plan.status = APPROXIFER_SEQUENCE_BAD;
    } else if (length > c.budget) {
        for (int j = thread; j < c.before(length); j += kT) {
            const int p = row[j];
            bad |= p < 0 || p >= c.P || c.refs[p < 0 || p >= c.P ? 0 : p] < 1;
        }
        plan.cut = 1;
    }
    if (plan.cut == 0) {                                      // all of it stays; what is refused keeps nothing that could be told
        for (int i = thread; i < c.budget; i += kT) kept[i] = plan.status == APPROXIFER_GROUP_OK && i < length ? i : -1;
        if (thread == 0) w.plans[b] = plan;
        return;
    }
    const float *const mass = c.mass + b * c.mass_stride;
    const int end = length - c.recent;
    const int moved = end - c.first <= kEach * kT ? select_kept<kT, true>(c, mass, row, end, kept, sources, bins, sums, found)
                                                  : select_kept<kT, false>(c, mass, row, end, kept, sources, bins, sums, found);
    if (__syncthreads_or(bad)) {                              // none of its pages has been looked into
        for (int i = thread; i < c.budget; i += kT) kept[i] = -1;
        plan.status = APPROXIFER_SEQUENCE_BAD_PAGE;
        plan.cut = 0;
        if (thread == 0) w.plans[b] = plan;
        return;
    }
    const int after = c.after();
    // a last page that is not full will be written to by who goes on: it changes hands even where its tokens stay
    plan.low = min(moved < c.budget ? moved >> c.shift : after, (c.budget & mask) != 0 ? c.budget >> c.shift : after);
    int32_t *const pages = w.pages + static_cast<int64_t>(b) * after;
    for (int j0 = plan.low; j0 < after; j0 += kT) {
        const int j = j0 + thread, p = j < after ? row[j] : 0;
        const bool wants = j < after && c.refs[p] > 1;
        int total;
        const int rank = plan.need + block_scan<int>(wants, sums, &total);
        if (j < after) pages[j] = wants ? -1 - rank : p;
        plan.need += total;
    }
    if (thread == 0) w.plans[b] = plan;
}

// 5 us for up to 64 sequences, most of it the launch and a chain of three loads.  Which pages are free is known when the call begins; a launch of
// its own, because where a sequence's begin in their list is the sum of what all before it want, which the launch before this one finds.  One workgroup:
// free pages, ascending, for the sequences in their order; where one finds too few, those behind it that want any do too.
__global__ __launch_bounds__(kThreads) void evict_pages_kernel(const int32_t *refs, EvictSpace w, int B, int P) {
    __shared__ int sums[16];
    __shared__ long long wide_sums[16];
    long long wanted = 0;
    for (int b0 = 0; b0 < B; b0 += kThreads) {
        const int b = b0 + threadIdx.x;
        long long total;
        block_scan<long long>(b < B ? w.plans[b].need : 0, wide_sums, &total);
        wanted += total;
    }
    if (wanted == 0) return;
    const int most = static_cast<int>(min(wanted, static_cast<long long>(P)));
    int available = 0;
    Stretch next;
    next.load(refs, 0, P);
    for (int at = 0; at < P && available < most; at += 4 * kThreads) {
        const Stretch now = next;
        next.load(refs, at + 4 * kThreads, P);
        int count = 0, total;
#pragma unroll
        for (int k = 0; k < 4; ++k) count += now.refs[k] == 0;
        int rank = available + block_scan(count, sums, &total);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (now.refs[k] == 0) {
                if (rank < most) w.list[rank] = at + 4 * static_cast<int>(threadIdx.x) + k;
                ++rank;
            }
        available = min(available + total, most);
    }
    long long upto = 0;
    for (int b0 = 0; b0 < B; b0 += kThreads) {
        const int b = b0 + threadIdx.x, need = b < B ? w.plans[b].need : 0;
        long long total;
        const long long start = upto + block_scan<long long>(need, wide_sums, &total);
        upto += total;
        if (need == 0) continue;
        if (start + need <= available) w.plans[b].offset = static_cast<int>(start);
        else w.plans[b].status = APPROXIFER_SEQUENCE_NO_PAGES;
    }
}

constexpr int kLoads = 4;                                     // pieces of 16 bytes that a thread has on their way
constexpr int kNoVmem = 0x0f70;                               // of s_waitcnt: until no load from memory is on its way

// 333 us for 1.6 GB (above).  Which places are read is looked up for the next stretch while this one's four pieces a thread are on their way, and
// all four are asked for without a branch between them: with both left to their order 1014 us.  The first `rows` workgroups bring
// the sequences up to date, the others copy: a head of a plane, or `pieces` of each of its rows, at a time.
__global__ __launch_bounds__(256) void evict_move_kernel(EvictCall c, EvictSpace w, char *pools, int64_t planes, int64_t heads,
                                                         int64_t row_bytes, int pieces, int rows) {
    const int thread = threadIdx.x, after = c.after(), mask = (1 << c.shift) - 1;
    const auto page_of = [&](const EvictPlan &plan, const int32_t *pages, int j) {
        const int p = pages[j];
        return p >= 0 ? p : w.list[plan.offset - 1 - p];
    };
    if (static_cast<int>(blockIdx.x) < rows) {
        for (int b = blockIdx.x; b < c.B; b += rows) {
            const EvictPlan plan = w.plans[b];
            int32_t *const kept = c.kept + static_cast<int64_t>(b) * c.budget, *const row = c.table + static_cast<int64_t>(b) * c.M;
            if (thread == 0 && c.status != nullptr) c.status[b] = plan.status;
            if (plan.status == APPROXIFER_SEQUENCE_NO_PAGES)
                for (int i = thread; i < c.budget; i += 256) kept[i] = -1;
            if (plan.status != APPROXIFER_GROUP_OK || plan.cut == 0) continue;
            const int32_t *const pages = w.pages + static_cast<int64_t>(b) * after;
            for (int j = plan.low + thread; j < c.before(plan.length); j += 256) {
                if (j < after && pages[j] >= 0) continue;
                atomicSub(&c.refs[row[j]], 1);                // integers: the order does not show
                const int p = j < after ? page_of(plan, pages, j) : -1;
                if (p >= 0) c.refs[p] = 1;
                row[j] = p;
            }
            if (thread == 0) c.lens[b] = c.budget;
            float *const mass = c.mass + b * c.mass_stride;
            for (int i0 = 0; i0 < c.budget; i0 += 256 * 8) {  // masses behind one of them are read before they are written
                float x[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = i0 + k * 256 + thread < c.budget ? mass[kept[i0 + k * 256 + thread]] : 0.0f;
                __builtin_amdgcn_s_waitcnt(kNoVmem);
                __syncthreads();
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (i0 + k * 256 + thread < c.budget) mass[i0 + k * 256 + thread] = x[k];
            }
            __syncthreads();
            for (int i = c.budget + thread; i < plan.length; i += 256) mass[i] = 0.0f;
        }
        return;
    }
    const int splits = static_cast<int>(row_bytes / 16 / pieces), size = 1 << c.shift;
    const int64_t items = c.B * planes * heads * splits;
    const int tokens = 256 * kLoads / pieces;                 // of a stretch: what a thread has of it never changes
    int token[kLoads], piece[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        const unsigned n = k * 256 + thread;
        token[k] = static_cast<int>(n / static_cast<unsigned>(pieces));
        piece[k] = static_cast<int>(n % static_cast<unsigned>(pieces));
    }
    for (int64_t item = blockIdx.x - rows; item < items; item += gridDim.x - rows) {
        const int part = static_cast<int>(item % splits);
        const int64_t head = item / splits % heads, plane = item / splits / heads % planes;
        const int b = static_cast<int>(item / splits / heads / planes);
        const EvictPlan plan = w.plans[b];
        if (plan.status != APPROXIFER_GROUP_OK || plan.cut == 0 || plan.low >= after) continue;
        const int32_t *const pages = w.pages + static_cast<int64_t>(b) * after;
        const int32_t *const kept = c.kept + static_cast<int64_t>(b) * c.budget, *const sources = w.sources + static_cast<int64_t>(b) * c.budget;
        const auto address = [&](int page, int slot, int piece) {
            return pools + (((plane * c.P + page) * heads + head) * size + slot) * row_bytes + (part * pieces + piece) * 16;
        };
        const int begin = plan.low << c.shift, last = c.budget - 1;
        const auto index = [&](int k, int i0) { return min(i0 + token[k], last); };
        int from[kLoads], slot[kLoads], to[kLoads];           // of the next stretch's pieces: asked for while this one's are on their way
        const auto look_up = [&](int i0) {
#pragma unroll
            for (int k = 0; k < kLoads; ++k) {
                const int i = index(k, i0);
                from[k] = sources[i];
                slot[k] = kept[i];
                to[k] = pages[i >> c.shift];
            }
            if (plan.need > 0) {
#pragma unroll
                for (int k = 0; k < kLoads; ++k) to[k] = to[k] >= 0 ? to[k] : w.list[plan.offset - 1 - to[k]];
            }
        };
        look_up(begin);
        for (int i0 = begin; i0 < c.budget; i0 += tokens) {
            v4f x[kLoads];
            char *at[kLoads];
#pragma unroll
            for (int k = 0; k < kLoads; ++k) {
                x[k] = *reinterpret_cast<const v4f *>(address(from[k], slot[k] & mask, piece[k]));
                at[k] = address(to[k], index(k, i0) & mask, piece[k]);
            }
            look_up(i0 + tokens);
            __builtin_amdgcn_s_waitcnt(kNoVmem);              // all that this stretch's tokens are written over has been read
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kLoads; ++k)
                if (token[k] < tokens && i0 + token[k] < c.budget) *reinterpret_cast<v4f *>(at[k]) = x[k];
        }
    }
}

int64_t rounded(int64_t ints) { return (ints + 63) / 64 * 64; }

}  // namespace

size_t evict_workspace_bytes(int64_t B, int64_t budget, int64_t P, int page_shift) {
    const int64_t after = (budget + (int64_t{1} << page_shift) - 1) >> page_shift;
    return static_cast<size_t>(4 * (rounded(B * static_cast<int64_t>(sizeof(EvictPlan) / 4)) + rounded(B * after) + rounded(B * budget) + rounded(P)));
}

int launch_cache_evict(int32_t *table, int32_t *lens, int32_t *refs, float *mass, int64_t mass_stride, int32_t *kept, int32_t *status,
                       void *pools, int64_t planes, int64_t heads, int64_t row_bytes, int B, int M, int P, int page_shift, int budget,
                       int first, int recent, void *workspace, hipStream_t stream) {
    const EvictCall c{table, lens, refs, mass, mass_stride, kept, status, B, M, P, page_shift, budget, first, recent};
    EvictSpace w;
    int32_t *const at = static_cast<int32_t *>(workspace);
    w.plans = static_cast<EvictPlan *>(workspace);
    w.pages = at + rounded(B * static_cast<int64_t>(sizeof(EvictPlan) / 4));
    w.sources = w.pages + rounded(static_cast<int64_t>(B) * c.after());
    w.list = w.sources + rounded(static_cast<int64_t>(B) * budget);
    // short sequences by fewer threads, which meet sooner
    const int64_t longest = mass_stride < static_cast<int64_t>(M) << page_shift ? mass_stride : static_cast<int64_t>(M) << page_shift;
    hipError_t e = longest <= 256 * kEach ? launch_kernel(evict_select_kernel<256>, dim3(B), dim3(256), 0, stream, c, w)
                                          : launch_kernel(evict_select_kernel<kThreads>, dim3(B), dim3(kThreads), 0, stream, c, w);
    if (e == hipSuccess) e = launch_kernel(evict_pages_kernel, dim3(1), dim3(kThreads), 0, stream, refs, w, B, P);
    if (e == hipSuccess) {
        // rows are cut, never below a sector of 64 bytes, until there is work for every CU; without pools there may be no piece in a row
        const int64_t whole = planes * heads * B, row = whole > 0 ? row_bytes / 16 : 1;
        int pieces = static_cast<int>(row);
        while (pieces % 2 == 0 && pieces >= 8 && whole * (row / pieces) < 1024) pieces /= 2;
        const int64_t items = whole * (row / pieces);
        const int rows = B < 1024 ? B : 1024;
        e = launch_kernel(evict_move_kernel, dim3(static_cast<unsigned>(rows + (items < 65536 ? items : 65536))), dim3(256), 0, stream, c, w,
                          static_cast<char *>(pools), planes, heads, row_bytes, pieces, rows);
    }
    return launch_status(e);
}

}  // namespace approxifer
