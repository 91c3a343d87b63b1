// The body of the tiles kernels, for a function with E, DP, kWhole, kSmall, kShared and c, g, workspace, shared, group_index, lds (attend_tiles.h).
// attend()'s kernel has it as its own: as a function in the kernel, inlined, it is simplified before the kernel's registers and arguments are
// known, and takes longer where heads are not whole (four prompts of 1000, 12 heads, bf16: of 48 31.5 us for 28.1, of 96 37.3 for 35.3).
    typedef typename E::Value V;
    typedef TileShape<E, DP> S;
    constexpr bool kDirect = kWhole && !kSmall && S::kStride == S::kPieces;
    constexpr int kKeys = S::kKeys, kBlocks = kKeys / 32, kSteps = S::kPieces / 2, kOut = DP / 32;
    constexpr int kVec = S::kSize == 2 ? 1 : kOut % 4 == 0 ? 4 : kOut % 2 == 0 ? 2 : 1;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), half = lane >> 5, row32 = lane & 31;
    const int group = c.Hq / c.Hkv;
    int part, index = 0, h, b;
    int64_t tile = 0;
    SharedUnit unit;
    if constexpr (kShared) {
        unit = shared_unit(c, shared, group_index, S::kRows);
        if (unit.rows == 0) return;
        part = unit.part;
        h = unit.h;
        b = unit.b;
        tile = unit.block;
    } else {
        const int64_t heads = g.slots * c.Hkv, work = heads * g.parts;
        if (blockIdx.x >= work) {                             // the last workgroups: statuses, a wave for each
            const int64_t b = (blockIdx.x - work) * S::kWaves + wave;
            if (b >= c.seq.B) return;
            const int st = attend_status(c, static_cast<int>(b));
            if (lane == 0) c.status[b] = st;
            return;
        }
        part = static_cast<int>(blockIdx.x / heads);
        index = static_cast<int>(blockIdx.x % heads);
        h = index % c.Hkv;
        const int64_t slot = g.slots - 1 - index / c.Hkv;
        b = g.single ? static_cast<int>(slot) : slot_owner(c.seq, slot, group, S::kRows, &tile);
    }
    Rows rows;
    if constexpr (!kShared) rows = rows_of(c.seq, b);
    const int64_t row_count = kShared ? unit.rows : static_cast<int64_t>(rows.n) * group, first = tile * S::kRows;
    if (!kShared && (!rows.ok || rows.n > c.max_rows || rows.length > c.max_len || tile < 0 || first >= row_count)) return;

    // this lane's row; lanes behind the last row repeat it
    const int64_t row = min(first + wave * 32 + row32, row_count - 1);
    const int token = static_cast<int>(row / group), head = h * group + static_cast<int>(row % group);
    const int64_t start = kShared ? unit.start : rows.start;
    int place, p0, p1, w0, w1;                                // places: this row's, and the least and largest of the tile and of the wave
    if constexpr (kShared) {
        place = shared_place(c, unit, start + token);
        unit.find_leader(c);
        b = unit.b;
        unit.places_of(place, S::kWaves, reinterpret_cast<int *>(lds), &p0, &p1, &w0, &w1);
    } else {
        place = rows.place(token);
        p0 = rows.place(static_cast<int>(first / group));
        p1 = rows.place(static_cast<int>(min(first + S::kRows - 1, row_count - 1) / group));
        w0 = __builtin_amdgcn_readfirstlane(place);
        w1 = __builtin_amdgcn_readlane(place, 31);
    }
    const int end = kShared ? unit.end : 0x7fffffff, low = kShared ? unit.low : 0;         // of the keys that there are here
    const int near = kShared ? min(place, end - 1) : place;   // the last that this row sees of them

    v4i q[kSteps];
    {
        const V *x = static_cast<const V *>(c.q) + (start + token) * c.q_stride + static_cast<int64_t>(head) * c.Dh;
        const bool whole = reinterpret_cast<uintptr_t>(c.q) % 16 == 0 && c.q_stride % S::kPerPiece == 0;
        const unsigned flip = c.scale < 0.0f ? (S::kSize == 4 ? 0x80000000u : 0x80008000u) : 0u;
        const int Dh = c.scale == 0.0f ? 0 : kWhole ? DP : c.Dh;  // scale 0: scores of 0 at scale 1
#pragma unroll
        for (int s = 0; s < kSteps; ++s) q[s] = query_piece<E>(x, (2 * s + half) * S::kPerPiece, Dh, whole, flip);
    }
    const float scale = c.scale == 0.0f ? 1.0f : fabsf(c.scale) * 1.44269504088896340736f;

    const KeyTiles<kKeys, kShared> keys(c.window, c.sinks, p0, p1, low, end);
    const int chunk = kShared ? unit.chunk_of<kKeys>(keys.steps) : g.chunk_of<kKeys>(keys.steps);
    const int begin = part * chunk, steps = min(keys.steps, begin + chunk);       // this part's tiles: begin .. steps - 1
    if (!kShared && begin >= steps && part > 0) return;
    if constexpr (kShared) {
        if (begin >= steps) {                                 // nothing here: who joins the rows does not look at their sums
            if (half == 0 && first + wave * 32 + row32 < row_count)
                shared.settle(c, unit.sum_part, (start + token) * c.Hq + head, -INFINITY, 0.0f);
            return;
        }
    }
    const bool alone = !kShared && keys.steps <= chunk;
    const auto begin_of = [&](int it) { return keys.begin_of(it); };
    const int32_t *table = c.seq.table + static_cast<int64_t>(b) * c.seq.M;
    const int shift = c.seq.page_shift, in_page = (1 << shift) - 1;
    const auto page_at = [&](int it) {                        // of key `lane` of the tile
        return table[keys.seen(begin_of(min(it, steps - 1)) + (lane & (kKeys - 1))) >> shift];
    };
    const V *const k_pool = static_cast<const V *>(c.k_pool), *const v_pool = static_cast<const V *>(c.v_pool);

    v4i k_next[S::kLoads], v_next[S::kLoads];
    unsigned long long bad_next = 0, bad = 0;
    int page_next = begin < steps ? page_at(begin) : 0;
    const int Dh = kWhole ? DP : c.Dh;
    const auto load = [&](int it) {                           // this wave's keys of tile `it` into registers
        const bool off = page_next < 0 || page_next >= c.seq.P;
        bad_next = __ballot(off);
        const int page = off ? 0 : page_next, j0 = begin_of(it) + wave * S::kOwn;
        const auto piece = [&](const V *x, int at) {
            v4i y = *reinterpret_cast<const v4i *>(x + (kWhole || at < Dh ? at : 0));
            if (!kWhole && at >= Dh) y = v4i{0, 0, 0, 0};     // values behind the head
            return y;
        };
        if constexpr (!kSmall) {                         // one page: the address is the wave's, plus a constant of the lane's
            const int p = __builtin_amdgcn_readlane(page, wave * S::kOwn);
            const int64_t base = ((static_cast<int64_t>(p) * c.Hkv + h) * (in_page + 1) + (j0 & in_page)) * Dh;
            const V *const k = k_pool + base, *const v = v_pool + base;
#pragma unroll
            for (int n = 0; n < S::kLoads; ++n) {
                const int index = n * kWave + lane, key = index / S::kPieces, at = index % S::kPieces * S::kPerPiece;
                k_next[n] = piece(k + key * Dh, at);
                v_next[n] = piece(v + key * Dh, at);
            }
        } else {
#pragma unroll
            for (int n = 0; n < S::kLoads; ++n) {
                const int index = n * kWave + lane, key = index / S::kPieces, at = index % S::kPieces * S::kPerPiece;
                const int p = __shfl(page, wave * S::kOwn + key);
                const int64_t base = ((static_cast<int64_t>(p) * c.Hkv + h) * (in_page + 1) + ((j0 + key) & in_page)) * Dh;
                k_next[n] = piece(k_pool + base, at);
                v_next[n] = piece(v_pool + base, at);
            }
        }
        page_next = page_at(it + 1);
    };
    // The same straight into LDS, without a register: LDS takes the lanes' 16 bytes one behind the other, so each lane asks for the piece that
    // the row's permutation has there.
    const auto fetch = [&](int it) {
        char *const kt = lds + (it & 1) * 2 * S::kBytes, *const vt = kt + S::kBytes;
        const bool off = page_next < 0 || page_next >= c.seq.P;
        bad_next = __ballot(off);
        const int page = off ? 0 : page_next, j0 = begin_of(it) + wave * S::kOwn;
        const int p = __builtin_amdgcn_readlane(page, wave * S::kOwn);
        const int64_t base = ((static_cast<int64_t>(p) * c.Hkv + h) * (in_page + 1) + (j0 & in_page)) * Dh;
#pragma unroll
        for (int n = 0; n < S::kLoads; ++n) {
            const int index = n * kWave + lane, key = index / S::kStride;
            const int at = key * Dh + ((index % S::kStride) ^ permuted<S::kStride>(wave * S::kOwn + key)) * S::kPerPiece;
            const int to = wave * S::kOwn * S::kStride * 16 + n * kWave * 16;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(k_pool + base + at),
                                             (__attribute__((address_space(3))) void *)(kt + to), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(v_pool + base + at),
                                             (__attribute__((address_space(3))) void *)(vt + to), 16, 0, 0);
        }
        page_next = page_at(it + 1);
    };
    const auto whole_tile = [&](int j0, int a, int b) {       // every row from place a to place b sees every key
        if (kShared && (j0 < low || j0 + kKeys > end)) return false;
        return j0 + kKeys - 1 <= a && (c.window == 0 || j0 > b - c.window || j0 + kKeys <= c.sinks);
    };
    const auto put = [&](int it) {                            // from the registers into LDS
        char *const kt = lds + (it & 1) * 2 * S::kBytes, *const vt = kt + S::kBytes;
        if (!whole_tile(begin_of(it), p0, p1)) {              // seen by nobody: whatever the page holds there
#pragma unroll
            for (int n = 0; n < S::kLoads; ++n) {
                const int j = begin_of(it) + wave * S::kOwn + (n * kWave + lane) / S::kPieces;
                if (keys.seen(j) != j) v_next[n] = v4i{0, 0, 0, 0};
            }
        }
#pragma unroll
        for (int n = 0; n < S::kLoads; ++n) {
            const int index = n * kWave + lane, key = wave * S::kOwn + index / S::kPieces, piece = index % S::kPieces;
            *reinterpret_cast<v4i *>(kt + S::at(key, piece)) = k_next[n];
            *reinterpret_cast<v4i *>(vt + S::at(key, piece)) = v_next[n];
        }
        bad = bad_next;
    };
    const auto settle = [&](int it) {                         // what fetch() brings is there, and cleared as put() does
        __builtin_amdgcn_s_waitcnt(kNoVmem);
        if (!whole_tile(begin_of(it), p0, p1)) {
            char *const vt = lds + (it & 1) * 2 * S::kBytes + S::kBytes + wave * S::kOwn * S::kStride * 16;
#pragma unroll
            for (int n = 0; n < S::kLoads; ++n) {
                const int index = n * kWave + lane, j = begin_of(it) + wave * S::kOwn + index / S::kStride;
                v4i *const at = reinterpret_cast<v4i *>(vt + index * 16);
                if (keys.seen(j) != j) *at = v4i{0, 0, 0, 0};
            }
        }
        bad = bad_next;
    };

    v16f out[kOut];
#pragma unroll
    for (int n = 0; n < kOut; ++n)
#pragma unroll
        for (int k = 0; k < 16; ++k) out[n][k] = 0.0f;
    float top = -INFINITY, total = 0.0f;

    if (begin < steps) {
        if constexpr (kDirect) {
            fetch(begin);
            settle(begin);
        } else {
            load(begin);
            put(begin);
        }
    }
    __syncthreads();
    for (int it = begin; it < steps; ++it) {
        const int j0 = begin_of(it);
        const unsigned long long bad_now = bad;
        if (it + 1 < steps) {
            if constexpr (kDirect) fetch(it + 1);
            else load(it + 1);
        }
        const char *const kt = lds + (it & 1) * 2 * S::kBytes, *const vt = kt + S::kBytes;
        const bool none = j0 > (kShared ? min(w1, end - 1) : w1) || (c.window > 0 && j0 + kKeys - 1 <= w0 - c.window && j0 >= c.sinks);
        if (!none) {
            v16f s[kBlocks];
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
#pragma unroll
                for (int k = 0; k < 16; ++k) s[b][k] = 0.0f;
#pragma unroll
                for (int n = 0; n < kSteps; ++n)
                    s[b] = multiply<E>(*reinterpret_cast<const v4i *>(kt + S::at(b * 32 + row32, 2 * n + half)), q[n], s[b]);
            }
            // the products one behind the other with kAhead operands on their way: left alone, each waits for its own read
            __builtin_amdgcn_sched_group_barrier(kDsRead, S::kAhead, 0);
#pragma unroll
            for (int n = 0; n < kBlocks * kSteps - S::kAhead; ++n) {
                __builtin_amdgcn_sched_group_barrier(kMfma, S::kSize == 4 ? 4 : 1, 0);
                __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(kMfma, S::kAhead * (S::kSize == 4 ? 4 : 1), 0);
            // what is hidden from a row: keys behind it, keys before its window; and keys of bad pages are no numbers.  Few tiles need any
            // of it, and hardly one needs all.
            const int reach = near - j0 - 4 * half;
            if (bad_now != 0) {
                const unsigned long long off = bad_now >> (4 * half);
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (off >> (b * 32 + 8 * (k / 4) + k % 4) & 1) s[b][k] = NAN;
            }
            if (kShared && j0 < low) {
                const int ahead = low - j0 - 4 * half;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int k = 0; k < 16; ++k) s[b][k] = b * 32 + 8 * (k / 4) + k % 4 >= ahead ? s[b][k] : -INFINITY;
            }
            if (j0 + kKeys - 1 > (kShared ? min(w0, end - 1) : w0)) {
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int k = 0; k < 16; ++k) s[b][k] = b * 32 + 8 * (k / 4) + k % 4 <= reach ? s[b][k] : -INFINITY;
            }
            if (c.window != 0 && j0 <= w1 - c.window && j0 + kKeys > c.sinks) {
                const int start = c.sinks - j0 - 4 * half, back = (kShared ? place - j0 - 4 * half : reach) - c.window;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const int key = b * 32 + 8 * (k / 4) + k % 4;
                        s[b][k] = key > back || key < start ? s[b][k] : -INFINITY;
                    }
            }
            float most = s[0][0];
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int k = 0; k < 16; ++k) most = fmaxf(most, s[b][k]);
            most = fmaxf(half_max(most), top);
            // the maximum moves only where it has grown by a factor of 256 in the weights: they stay below that, and within their types
            if (__any((most - top) * scale > 8.0f)) {
                const float f = most == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((top - most) * scale);
                total *= f;
#pragma unroll
                for (int n = 0; n < kOut; ++n)
#pragma unroll
                    for (int k = 0; k < 16; ++k) out[n][k] *= f;
                top = most;
            }
            const float base = top == -INFINITY ? 0.0f : top * scale - kLift<E>;
            float sum = 0.0f;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    s[b][k] = __builtin_amdgcn_exp2f(fmaf(s[b][k], scale, -base));
                    sum += s[b][k];
                }
            total += sum;
            if constexpr (S::kSize == 2) {
                // weights in one piece of their type, at 2.1e-3 (bf16) and 2.7e-4 (fp16) of the outputs' norm from 64 bits; in two pieces, as the
                // few-rows kernel has them, 1.6e-3 and 2.0e-4, as the result's own rounding, but the two prompts of bf16 take 884 us
                // instead of 671 and the window of fp16 265 instead of 198
                const int i = lane & 15, quad = lane >> 4 & 1;
#pragma unroll
                for (int n = 0; n < kKeys / 16; ++n) {
                    float w[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) w[k] = s[n / 2][8 * (n % 2) + k];
                    const v4i p = rounded8<E>(w);
#pragma unroll
                    for (int o = 0; o < kOut; ++o) {
                        v4s x[2];
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const int key = 16 * n + 8 * u + 4 * half + (i >> 2);
                            const char *a = vt + S::at(key, 4 * o + 2 * quad + (i >> 1 & 1)) + (i & 1) * 8;
                            x[u] = load_transposed(a);
                        }
                        const v8s y = __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
                        out[o] = multiply<E>(__builtin_bit_cast(v4i, y), p, out[o]);
                    }
                }
                // as above, with the weights of the next 16 keys between the products of these
                __builtin_amdgcn_sched_group_barrier(kDsRead, 6, 0);
#pragma unroll
                for (int n = 0; n < kKeys / 16 * kOut; ++n) {
                    __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(kDsRead, 2, 0);
                }
            } else {
                // a lane reads kVec neighbouring values of a key at once: they are its operands of kVec products, whose rows are every
                // kVec-th dimension
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const int key = b * 32 + 8 * (k / 4) + 4 * half + k % 4;
#pragma unroll
                        for (int o = 0; o < kOut; o += kVec) {
                            typedef float VV __attribute__((ext_vector_type(kVec)));
                            const int at = 32 * o + kVec * row32;
                            const VV x = *reinterpret_cast<const VV *>(vt + S::at(key, at >> 2) + (at & 3) * 4);
#pragma unroll
                            for (int e = 0; e < kVec; ++e)
                                out[o + e] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], s[b][k], out[o + e], 0, 0, 0);
                        }
                    }
            }
        }
        if (it + 1 < steps) {
            if constexpr (kDirect) settle(it + 1);
            else put(it + 1);
        }
        __syncthreads();
    }

    float *const partial = kShared ? nullptr : workspace + (index * static_cast<int64_t>(g.parts) + part) * part_floats(S::kRows, c.Dh);
    total = half_sum(total);
    if (!kShared && c.stats != nullptr && alone && half == 0 && first + wave * 32 + row32 < row_count)
        RowStats(top == -INFINITY ? top : top * scale - kLift<E>, total).store(c, start + token, head);
    // A weight of 0 (hidden, or rounded to it) times an infinity is NaN, and so is all that a hidden NaN touches: the product cannot hide it.
    // Rows with such sums are computed again, element by element; those whose weights are no numbers are NaN as they have to be.  (A prompt of 2048
    // tokens, 8 heads of 128 on 2, bf16: 0.08 to 0.1 ms, with an infinity that all rows see too; with a NaN in their place, where all rows are
    // computed again, 8.6 ms.)
    bool odd = false;
#pragma unroll
    for (int o = 0; o < kOut; ++o)
#pragma unroll
        for (int k = 0; k < 16; ++k) odd |= out[o][k] != out[o][k];
    const unsigned long long odd_lanes = __ballot(odd && total == total);
    const unsigned odd_rows = static_cast<unsigned>(odd_lanes | odd_lanes >> 32);
    if (first + wave * 32 + row32 < row_count && (odd_rows >> row32 & 1) == 0) {
        const float inverse = !alone ? 1.0f : total == 0.0f ? 0.0f : 1.0f / total;
        const int n = wave * 32 + row32;
        const int64_t at = (start + token) * c.Hq + head;
        float *sums = kShared ? shared.sums(c, unit.sum_part, at) : partial + n * c.Dh;
        if (!alone && half == 0) {
            const float most = top == -INFINITY ? top : top * scale - kLift<E>;
            if constexpr (kShared) {
                shared.settle(c, unit.sum_part, at, most, total);
            } else {
                partial[S::kRows * c.Dh + n] = most;
                partial[S::kRows * c.Dh + S::kRows + n] = total;
            }
        }
        V *y = static_cast<V *>(c.out) + at * c.Dh;
#pragma unroll
        for (int o = 0; o < kOut; o += kVec)
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < kVec; ++j) {              // values 4 j ..+3 of the 4 kVec that lie next to each other
                    const int d = 32 * o + kVec * (8 * k + 4 * half) + 4 * j;
                    const auto value = [&](int n) { return out[o + (4 * j + n) % kVec][4 * k + (4 * j + n) / kVec] * inverse; };
                    if (!kWhole && d >= c.Dh) continue;
                    if (alone) store4<E>(y + d, value(0), value(1), value(2), value(3));
                    else *reinterpret_cast<v4f *>(sums + d) = v4f{value(0), value(1), value(2), value(3)};
                }
    }
    float *const scratch = reinterpret_cast<float *>(lds) + wave * APPROXIFER_MAX_HEAD_DIM;      // the tiles are done with
    for (unsigned left = odd_rows; left != 0; left &= left - 1) {
        const int n = wave * 32 + __builtin_ctz(left);
        if (first + n >= row_count) continue;
        if constexpr (kShared) shared_part<E>(c, shared, unit, first + n, scratch, keys, begin, steps);
        else attend_part<E>(c, rows, first + n, h, scratch, keys, begin, steps, alone, partial, S::kRows, n);
    }
