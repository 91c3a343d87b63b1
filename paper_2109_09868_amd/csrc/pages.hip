// The pages of a cache: taken, shared, copied, given back and moved together.  All bookkeeping is on the device, so that no call
// waits for the host and every call can be captured; pages are given out in ascending order, so that results do not depend on
// which wave came first.
// Reserving is one workgroup's chain of loads and scans: 192 sequences, 32768 pages, 8 us as long as what is wanted is found in the first 4096
// entries, 1 us more for every 4096 behind them (192 pages wanted of 200 that are free: 15 us in 32648 pages, 72 in 259592); forking (8 prompts to 192 sequences, 193 MB moved) 40 to
// 42 us and compacting (932 MB moved) 195 to 198 us are bound by the copies: 4.7 TB/s, as a large copy.
#include "sequences.h"

namespace approxifer {

namespace {

constexpr int kThreads = 1024;                                // of the kernels that give out pages: one workgroup
constexpr int kList = 8192;                                   // free pages found at a time, in LDS

// Exclusive prefix sum over the workgroup, and the total; `sums` holds 16 of LDS.
template <class T>
__device__ __forceinline__ T block_scan(T v, T *sums, T *total) {
    const int lane = lane_id(), wave = wave_id(), waves = blockDim.x / kWave;
    T up = v;
    for (int o = 1; o < kWave; o <<= 1) {
        const T x = __shfl_up(up, o);
        if (lane >= o) up += x;
    }
    __syncthreads();                                          // the sums of the call before have been read
    if (lane == kWave - 1) sums[wave] = up;
    __syncthreads();
    if (wave == 0) {
        T x = lane < waves ? sums[lane] : 0;
        for (int o = 1; o < 16; o <<= 1) {
            const T y = __shfl_up(x, o);
            if (lane >= o) x += y;
        }
        if (lane < waves) sums[lane] = x;
    }
    __syncthreads();
    *total = sums[waves - 1];
    return up - v + (wave > 0 ? sums[wave - 1] : 0);
}

// The first `most` (at most kList) free pages from *cursor on, ascending, into list; how many there are.  Afterwards *cursor is
// where to go on once those have been taken.  By the whole workgroup of kThreads.  `ahead` holds the stretch's refs: those of the
// cursor on entry.
struct Stretch {
    int32_t refs[4];
    __device__ __forceinline__ void load(const int32_t *from, int at, int P) {
        const int p = at + 4 * static_cast<int>(threadIdx.x);
#pragma unroll
        for (int k = 0; k < 4; ++k) refs[k] = p + k < P ? from[p + k] : 1;
    }
};
__device__ __forceinline__ int find_free(const int32_t *refs, int P, int most, int *list, int *sums, int *cursor, Stretch ahead) {
    int found = 0, at = *cursor;
    while (found < most && at < P) {
        const int p0 = at + 4 * static_cast<int>(threadIdx.x);
        bool is_free[4];
        int count = 0;
        for (int k = 0; k < 4; ++k) {
            is_free[k] = ahead.refs[k] == 0;
            count += is_free[k];
        }
        ahead.load(refs, at + 4 * kThreads, P);
        int total;
        int rank = found + block_scan(count, sums, &total);
        for (int k = 0; k < 4; ++k)
            if (is_free[k]) {
                if (rank < most) list[rank] = p0 + k;
                ++rank;
            }
        found += total;
        if (found <= most) at += 4 * kThreads;                // else the rest of this stretch is for the next time
    }
    *cursor = at;
    __syncthreads();
    return min(found, most);
}

// What sequence b wants of approxifer_cache_reserve(): pages, or a status of its own.
struct Wish {
    int old_pages, pages, length, status;
};
__device__ __forceinline__ Wish wish_of(const int32_t *table, const int32_t *lens, const int32_t *refs, const int32_t *add, int b,
                                        int M, int P, int shift) {
    Wish w{0, 0, 0, APPROXIFER_GROUP_OK};
    const int l = lens[b], a = add[b], mask = (1 << shift) - 1;
    if (l < 0 || a < 0 || l + static_cast<int64_t>(a) > (static_cast<int64_t>(M) << shift)) {
        w.status = APPROXIFER_SEQUENCE_BAD;
        return w;
    }
    w.length = l + a;
    w.old_pages = static_cast<int>((static_cast<int64_t>(l) + mask) >> shift);
    if ((l & mask) != 0 && a > 0) {
        const int p = table[static_cast<int64_t>(b) * M + (l >> shift)];
        if (p < 0 || p >= P) w.status = APPROXIFER_SEQUENCE_BAD_PAGE;
        else if (refs[p] > 1) w.status = APPROXIFER_SEQUENCE_SHARED_PAGE;
        if (w.status != APPROXIFER_GROUP_OK) return w;
    }
    w.pages = static_cast<int>((static_cast<int64_t>(w.length) + mask) >> shift) - w.old_pages;
    return w;
}

// One workgroup.  The pages wanted are counted, as many free ones are looked up, and given to the sequences by their prefix sum.
__global__ __launch_bounds__(kThreads) void cache_reserve_kernel(int32_t *table, int32_t *lens, int32_t *refs, const int32_t *add,
                                                                 int32_t *status, int B, int M, int P, int shift) {
    __shared__ int list[kList];
    __shared__ int sums[16];
    __shared__ long long wide_sums[16];                       // wishes of 1024 sequences may pass 2^31 together
    long long wanted = 0;
    Stretch ahead;
    ahead.load(refs, 0, P);                                   // on its way while the sequences are looked at
    Wish mine{0, 0, 0, 0};                                    // of the first 1024 sequences: not looked up again
    for (int b0 = 0; b0 < B; b0 += kThreads) {
        const int b = b0 + threadIdx.x;
        const Wish w = b < B ? wish_of(table, lens, refs, add, b, M, P, shift) : Wish{0, 0, 0, 0};
        if (b0 == 0) mine = w;
        long long total;
        block_scan<long long>(w.pages, wide_sums, &total);
        wanted += total;
    }
    const int most = static_cast<int>(min(wanted, static_cast<long long>(P)));
    int available = most;                                     // free pages, as far as they are wanted
    int cursor = 0;
    if (most > kList) {                                       // more than one list: whether a sequence gets any must be known first
        available = 0;
        for (int p0 = 0; p0 < P; p0 += kThreads) {
            const int p = p0 + threadIdx.x;
            available += __syncthreads_count(p < P && refs[p] == 0);
        }
        available = min(available, most);
    }
    int from = 0;                                             // pages given out in the rounds before
    do {
        const int found = find_free(refs, P, min(most - from, kList), list, sums, &cursor, ahead);
        if (most <= kList) available = found;
        const bool last = from + found >= available;
        long long upto = 0;
        for (int b0 = 0; b0 < B; b0 += kThreads) {
            const int b = b0 + threadIdx.x;
            Wish w{0, 0, 0, 0};
            if (b0 == 0) w = mine;
            else if (b < B) w = wish_of(table, lens, refs, add, b, M, P, shift);
            long long total;
            const long long start = upto + block_scan<long long>(w.pages, wide_sums, &total);
            upto += total;
            const bool enough = start + w.pages <= available;
            if (enough)
                for (int k = static_cast<int>(max(0LL, from - start)); k < w.pages && start + k < from + found; ++k) {
                    const int p = list[start + k - from];
                    table[static_cast<int64_t>(b) * M + w.old_pages + k] = p;
                    refs[p] = 1;
                }
            if (last && b < B) {
                const int st = w.status != APPROXIFER_GROUP_OK ? w.status
                               : enough || w.pages == 0        ? APPROXIFER_GROUP_OK
                                                               : APPROXIFER_SEQUENCE_NO_PAGES;
                if (status != nullptr) status[b] = st;
                if (st == APPROXIFER_GROUP_OK) lens[b] = w.length;
            }
        }
        from += found;
        if (last) break;
        __syncthreads();
        ahead.load(refs, cursor, P);
    } while (true);
}

// ---- fork -------------------------------------------------------------------------------------------------------------
// Workspace: claims [P], sources [B_out], targets [B_out], the number of copies.
struct ForkSpace {
    int32_t *claims, *sources, *targets, *copies;
};
constexpr int kNobody = 0x7fffffff;

__global__ __launch_bounds__(256) void fork_begin_kernel(const int32_t *refs, int32_t *refs_out, int32_t *claims, int P) {
    const int p = blockIdx.x * 256 + threadIdx.x;
    if (p >= P) return;
    refs_out[p] = refs[p];
    claims[p] = kNobody;
}

// Blocks 0..B-1 take the old sequences' holds off, the others put the new ones' on full pages and say who wants a page that is not
// full.  Sums and minima of integers: the order of the atomics does not show.
__global__ __launch_bounds__(256) void fork_rows_kernel(const int32_t *table, const int32_t *lens, const int32_t *parents,
                                                        const int32_t *keep, int32_t *table_out, int32_t *lens_out,
                                                        int32_t *refs_out, int32_t *status, int32_t *claims, int B, int B_out, int M,
                                                        int P, int shift) {
    const int64_t most = static_cast<int64_t>(M) << shift;
    const int mask = (1 << shift) - 1;
    if (static_cast<int>(blockIdx.x) < B) {
        const int b = blockIdx.x, l = lens[b];
        if (l < 0 || l > most) return;
        const int pages = static_cast<int>((static_cast<int64_t>(l) + mask) >> shift);
        for (int j = threadIdx.x; j < pages; j += 256) {
            const int p = table[static_cast<int64_t>(b) * M + j];
            if (p >= 0 && p < P) atomicSub(&refs_out[p], 1);
        }
        return;
    }
    const int i = blockIdx.x - B, r = parents[i];
    int st = APPROXIFER_GROUP_OK, l = 0;
    if (r < -1 || r >= B || (keep != nullptr && keep[i] < 0)) st = APPROXIFER_SEQUENCE_BAD;
    else if (r >= 0) {
        l = lens[r];
        if (l < 0 || l > most) st = APPROXIFER_SEQUENCE_BAD;
        else if (keep != nullptr) l = min(l, keep[i]);
    }
    if (st != APPROXIFER_GROUP_OK) l = 0;
    const int32_t *row = table + static_cast<int64_t>(max(r, 0)) * M;   // read only where l > 0
    int32_t *out = table_out + static_cast<int64_t>(i) * M;
    const int pages = static_cast<int>((static_cast<int64_t>(l) + mask) >> shift);
    bool bad = false;
    for (int j = threadIdx.x; j < pages; j += 256) bad |= row[j] < 0 || row[j] >= P;
    if (__syncthreads_or(bad)) {
        st = APPROXIFER_SEQUENCE_BAD_PAGE;
        l = 0;
    }
    const int full = l >> shift;
    for (int j = threadIdx.x; j < M; j += 256) {
        int p = -1;
        if (j < full) {
            p = row[j];
            atomicAdd(&refs_out[p], 1);
        } else if (j == full && (l & mask) != 0) {
            p = row[j];
            atomicMin(&claims[p], i);
        }
        out[j] = p;
    }
    if (threadIdx.x == 0) {
        lens_out[i] = l;
        if (status != nullptr) status[i] = st;
    }
}

// One workgroup: who takes a page over, and a free page for everybody else who wants one.
__global__ __launch_bounds__(kThreads) void fork_pages_kernel(int32_t *table_out, int32_t *lens_out, int32_t *refs_out,
                                                              int32_t *status, ForkSpace w, int B_out, int M, int P, int shift) {
    __shared__ int list[kList];
    __shared__ int sums[16];
    const int mask = (1 << shift) - 1;
    int wanted = 0;
    for (int i0 = 0; i0 < B_out; i0 += kThreads) {
        const int i = i0 + threadIdx.x;
        bool copies = false;
        if (i < B_out) {
            const int l = lens_out[i];
            if ((l & mask) != 0) {
                const int p = table_out[static_cast<int64_t>(i) * M + (l >> shift)];
                copies = true;
                if (w.claims[p] == i && refs_out[p] == 0) {   // nobody else passes the first test
                    w.claims[p] = -2 - i;
                    refs_out[p] = 1;
                    copies = false;
                }
            }
        }
        wanted += __syncthreads_count(copies);
    }
    __syncthreads();
    int cursor = 0, from = 0;
    while (true) {
        Stretch ahead;
        ahead.load(refs_out, cursor, P);
        const int found = find_free(refs_out, P, min(wanted - from, kList), list, sums, &cursor, ahead);
        const bool last = from + found >= wanted || found < kList;
        int upto = 0;
        for (int i0 = 0; i0 < B_out; i0 += kThreads) {
            const int i = i0 + threadIdx.x;
            int p = -1, l = 0;
            if (i < B_out) {
                l = lens_out[i];
                if ((l & mask) != 0) {
                    p = table_out[static_cast<int64_t>(i) * M + (l >> shift)];
                    if (w.claims[p] == -2 - i) p = -1;
                }
            }
            // one that a round before has served has its target in the table: its rank, not its page, says so
            const bool copies = p >= 0;
            int total;
            const int rank = upto + block_scan<int>(copies, sums, &total);
            upto += total;
            if (copies && rank >= from && rank < from + found) {
                const int target = list[rank - from];
                w.sources[rank] = p;
                w.targets[rank] = target;
                refs_out[target] = 1;
            }
            if (copies && last) {
                int32_t *row = table_out + static_cast<int64_t>(i) * M;
                if (rank < from + found) {
                    row[l >> shift] = rank >= from ? list[rank - from] : w.targets[rank];
                } else {                                      // no page left: an empty sequence that holds nothing
                    for (int j = 0; j < (l >> shift); ++j) {
                        atomicSub(&refs_out[row[j]], 1);
                        row[j] = -1;
                    }
                    row[l >> shift] = -1;
                    lens_out[i] = 0;
                    if (status != nullptr) status[i] = APPROXIFER_SEQUENCE_NO_PAGES;
                }
            }
        }
        from += found;
        if (last) break;
        __syncthreads();
    }
    if (threadIdx.x == 0) *w.copies = from;
}

// ---- copies of pages ----------------------------------------------------------------------------------------------------
constexpr int kPiece = 16384;                                 // bytes that a workgroup of 256 copies at once

// Pieces of `copies` pages in all planes, `block` of `blocks` workgroups.
__device__ void copy_pages(const int32_t *sources, const int32_t *targets, int copies, char *pools, int64_t planes,
                           int64_t page_bytes, int P, int64_t block, int64_t blocks) {
    const int64_t pieces = (page_bytes + kPiece - 1) / kPiece, items = copies * planes * pieces;
    for (int64_t n = block; n < items; n += blocks) {
        const int64_t piece = n % pieces, plane = n / pieces % planes, m = n / pieces / planes;
        const char *from = pools + (plane * P + sources[m]) * page_bytes;
        char *to = pools + (plane * P + targets[m]) * page_bytes;
        const int64_t at = piece * kPiece + threadIdx.x * 16;
        v4f x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (at + k * 4096 < page_bytes) x[k] = *reinterpret_cast<const v4f *>(from + at + k * 4096);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (at + k * 4096 < page_bytes) *reinterpret_cast<v4f *>(to + at + k * 4096) = x[k];
    }
}

__global__ __launch_bounds__(256) void fork_copy_kernel(ForkSpace w, char *pools, int64_t planes, int64_t page_bytes, int P) {
    copy_pages(w.sources, w.targets, *w.copies, pools, planes, page_bytes, P, blockIdx.x, gridDim.x);
}

// ---- compact ------------------------------------------------------------------------------------------------------------
// Workspace: live pages of each segment, sources and targets [P / 2], the number of moves.
constexpr int kSegment = 1024;
struct CompactSpace {
    int32_t *counts, *sources, *targets, *moves;
};

__global__ __launch_bounds__(kSegment) void compact_count_kernel(const int32_t *refs, int32_t *counts, int P) {
    const int p = blockIdx.x * kSegment + threadIdx.x;
    const int n = __syncthreads_count(p < P && refs[p] != 0);
    if (threadIdx.x == 0) counts[blockIdx.x] = n;
}

// A workgroup per segment: rank of every live page behind the line and of every free place before it.  A moving page's entry of
// `moved` holds -2 - rank until the next kernel.
__global__ __launch_bounds__(kSegment) void compact_rank_kernel(const int32_t *refs, int32_t *moved, int32_t *live_out, CompactSpace w,
                                                                int P) {
    __shared__ int sums[16];
    const int segment = blockIdx.x, segments = gridDim.x;
    int before = 0, live = 0, total;
    for (int s0 = 0; s0 < segments; s0 += kSegment) {
        const int s = s0 + threadIdx.x, n = s < segments ? w.counts[s] : 0;
        block_scan(n, sums, &total);
        live += total;
        block_scan(s < segment ? n : 0, sums, &total);
        before += total;
    }
    // live pages before the line: those of whole segments, and of the piece that it cuts
    int below = 0;
    for (int s0 = 0; s0 < segments; s0 += kSegment) {
        const int s = s0 + threadIdx.x;
        block_scan(s < live / kSegment ? w.counts[s] : 0, sums, &total);
        below += total;
    }
    const int cut = live / kSegment * kSegment + threadIdx.x;
    below += __syncthreads_count(cut < live && refs[cut] != 0);
    const int p = segment * kSegment + threadIdx.x;
    const bool alive = p < P && refs[p] != 0;
    const int rank = before + block_scan<int>(alive, sums, &total);      // live pages before p
    if (p < P) {
        int to = alive ? p : -1;
        if (alive && p >= live) {
            w.sources[rank - below] = p;
            to = -2 - (rank - below);
        }
        if (!alive && p < live) w.targets[p - rank] = p;
        moved[p] = to;
    }
    if (segment == 0 && threadIdx.x == 0) {
        *live_out = live;
        *w.moves = live - below;
    }
}

// The first `rows` workgroups bring tables, refs and `moved` up to date, the others copy.
__global__ __launch_bounds__(256) void compact_move_kernel(int32_t *table, const int32_t *lens, int32_t *refs, int32_t *moved,
                                                           CompactSpace w, char *pools, int64_t planes, int64_t page_bytes, int B, int M,
                                                           int P, int shift, int rows) {
    const int moves = *w.moves;
    if (static_cast<int>(blockIdx.x) >= rows) {
        copy_pages(w.sources, w.targets, moves, pools, planes, page_bytes, P, blockIdx.x - rows, gridDim.x - rows);
        return;
    }
    for (int m = blockIdx.x * 256 + threadIdx.x; m < moves; m += rows * 256) {
        const int from = w.sources[m], to = w.targets[m];
        refs[to] = refs[from];
        refs[from] = 0;
        moved[from] = to;                                     // readers below take the rank or the target, whichever they find
    }
    const int64_t most = static_cast<int64_t>(M) << shift;
    for (int b = blockIdx.x; b < B; b += rows) {
        const int l = lens[b];
        if (l < 0 || l > most) continue;
        const int pages = static_cast<int>((static_cast<int64_t>(l) + (1 << shift) - 1) >> shift);
        for (int j = threadIdx.x; j < pages; j += 256) {
            int32_t *at = table + static_cast<int64_t>(b) * M + j;
            const int p = *at;
            if (p < 0 || p >= P) continue;
            const int to = moved[p];
            if (to < -1) *at = w.targets[-2 - to];
            else if (to >= 0 && to != p) *at = to;
        }
    }
}

int64_t rounded(int64_t ints) { return (ints * 4 + 255) / 256 * 64; }

unsigned copy_blocks(int64_t most_copies, int64_t planes, int64_t page_bytes) {
    const int64_t items = most_copies * planes * ((page_bytes + kPiece - 1) / kPiece);
    return static_cast<unsigned>(items < 2048 ? items : 2048);
}

}  // namespace

size_t cache_workspace_bytes(int64_t B, int64_t B_out, int64_t P) {
    (void)B;
    const int64_t fork = rounded(P) + 2 * rounded(B_out), compact = rounded((P + kSegment - 1) / kSegment) + 2 * rounded(P / 2 + 1);
    return static_cast<size_t>(4 * ((fork > compact ? fork : compact) + 64));
}

int launch_cache_reserve(int32_t *table, int32_t *lens, int32_t *refs, const int32_t *add, int32_t *status, int B, int M, int P,
                         int page_shift, hipStream_t stream) {
    return launch_status(launch_kernel(cache_reserve_kernel, dim3(1), dim3(kThreads), 0, stream, table, lens, refs, add, status, B, M,
                                       P, page_shift));
}

int launch_cache_fork(const int32_t *table, const int32_t *lens, const int32_t *refs, const int32_t *parents, const int32_t *keep,
                      int32_t *table_out, int32_t *lens_out, int32_t *refs_out, int32_t *status, void *pools, int64_t planes,
                      int64_t page_bytes, int B, int B_out, int M, int P, int page_shift, void *workspace, hipStream_t stream) {
    ForkSpace w;
    w.copies = static_cast<int32_t *>(workspace);
    w.claims = w.copies + 64;
    w.sources = w.claims + rounded(P);
    w.targets = w.sources + rounded(B_out);
    hipError_t e = hipSuccess;
    if (P > 0) e = launch_kernel(fork_begin_kernel, dim3((P + 255) / 256), dim3(256), 0, stream, refs, refs_out, w.claims, P);
    if (e == hipSuccess && static_cast<int64_t>(B) + B_out > 0)
        e = launch_kernel(fork_rows_kernel, dim3(static_cast<unsigned>(B) + static_cast<unsigned>(B_out)), dim3(256), 0, stream, table,
                          lens, parents, keep, table_out, lens_out, refs_out, status, w.claims, B, B_out, M, P, page_shift);
    if (e == hipSuccess && B_out > 0 && P > 0) {
        e = launch_kernel(fork_pages_kernel, dim3(1), dim3(kThreads), 0, stream, table_out, lens_out, refs_out, status, w, B_out, M, P,
                          page_shift);
        const unsigned blocks = copy_blocks(B_out, planes, page_bytes);
        if (e == hipSuccess && blocks > 0)
            e = launch_kernel(fork_copy_kernel, dim3(blocks), dim3(256), 0, stream, w, static_cast<char *>(pools), planes, page_bytes,
                              P);
    }
    return launch_status(e);
}

int launch_cache_compact(int32_t *table, const int32_t *lens, int32_t *refs, int32_t *moved, int32_t *live, void *pools,
                         int64_t planes, int64_t page_bytes, int B, int M, int P, int page_shift, void *workspace,
                         hipStream_t stream) {
    const int segments = (P + kSegment - 1) / kSegment;
    CompactSpace w;
    w.moves = static_cast<int32_t *>(workspace);
    w.counts = w.moves + 64;
    w.sources = w.counts + rounded(segments);
    w.targets = w.sources + rounded(P / 2 + 1);
    hipError_t e = launch_kernel(compact_count_kernel, dim3(segments), dim3(kSegment), 0, stream, refs, w.counts, P);
    if (e == hipSuccess)
        e = launch_kernel(compact_rank_kernel, dim3(segments), dim3(kSegment), 0, stream, refs, moved, live, w, P);
    if (e == hipSuccess) {
        const int rows = B < 1 ? 1 : B < 256 ? B : 256;
        const unsigned blocks = copy_blocks(P / 2, planes, page_bytes);
        e = launch_kernel(compact_move_kernel, dim3(rows + blocks), dim3(256), 0, stream, table, lens, refs, moved, w,
                          static_cast<char *>(pools), planes, page_bytes, B, M, P, page_shift, rows);
    }
    return launch_status(e);
}

}  // namespace approxifer
