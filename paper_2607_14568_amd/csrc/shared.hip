// Paged attention of a batch whose sequences share long prefixes (included by gdn.hip, behind paged.hip, whose kernels it runs).
//
// The sequences of a group hold the same first P tokens in the same pages.  With softmax weights relative to any reference,
// a row's output over all its keys is the weighted mean of those over the prefix and over what is behind it:
//   m = max(m1, m2),  l = l1 2^(m1 - m) + l2 2^(m2 - m),  o = (o1 2^(m1 - m) + o2 2^(m2 - m)) / l.
// The rows of all the group's new tokens attend the prefix together (each sees all of it, so no key is masked), which reads
// it once for the group, and every sequence's rows attend its own keys behind it.  So one call takes
//   k_shared_setup   more than 64 sequences: the parts, groups and sequences with their keys, chunks and items, from the lengths on
//                    the device (up to 64, a lane each, every wave of the next one does so by itself: 8, 32 and 64 sequences
//                    take 19.0, 34.3 and 52.5 us so, 21.9, 37.0 and 55.5 with this kernel)
//   k_attn_shared    the items, of the groups' prefixes (first in the grid) and of the sequences' own keys, by the workgroups of
//                    k_attn_rows and k_attn_tile
//   k_shared_join    every row's partial sums added up in order
// A sequence that does not reach behind its group's prefix (a finished one, one that does not belong) takes no part in it and
// attends all its keys by itself.

// Inclusive sums over the wave's lanes, as wave_scan takes them: always in the same order.
template <int CTRL, int ROWS> __device__ __forceinline__ double dpp64(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xf, false);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double scan64(double x) {
    x += dpp64<0x111, 0xf>(x);
    x += dpp64<0x112, 0xf>(x);
    x += dpp64<0x114, 0xf>(x);
    x += dpp64<0x118, 0xf>(x);
    x += dpp64<0x142, 0xa>(x);
    x += dpp64<0x143, 0xc>(x);
    return x;
}
__device__ __forceinline__ double lane64(double x, int l) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)u, l), hi = __builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), l);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

struct SharedParams : PagedParams {
    const int32_t* prefix;    // [groups] tokens that a group's sequences share
    const int32_t* cu_groups; // [groups + 1] offsets of the groups among the sequences; null: one group
    int groups;
    int rbp, rbt;             // rows per block of the prefixes and of the sequences' own keys (round: items at once, of both)
    // The parts as k_shared_setup left them, or null: up to 64 sequences, whose parts every wave works out by itself.
    const int4* part;         // groups {first token, tokens, P, a sequence that shares}, or sequences {first token, tokens, length, start}
    const int32_t* first;     // [parts + 1] items of one key/value head ahead of each part's
    const int32_t* chunk;     // units per chunk (one word)
    int parts;
    bool of_prefix;           // the groups' prefixes, or the sequences' own keys
};

// Units per chunk, of prefixes and own keys alike: an even share of all row blocks' units for each item that is resident at once,
// `round` of them.  That makes at most round + (row blocks) items (ceil(u / c) < u / c + 1): those past the round, mostly short
// sequences, start as others end.  (A c that makes at most `round` items leaves too few of the long ones where there are many
// short: 32 sequences behind 65536 tokens, e4m3, 76.8 us against 57.7.  A prefix's unit counted as two of a sequence's,
// since its 128 rows take longer: 55 against 52.4 for 64 sequences behind 8192.)
__device__ __forceinline__ int chunk_units(double all, int round) { return max((int)min(ceil(all / round), 0x1p23), 1); }

// What k_shared_join takes of a sequence, and where its row blocks begin (of one key/value head).
struct SharedNote {
    int tok, n, len, start;           // first token, tokens, length, first key of its own
    int first, block, c, gfirst;      // first item; first row block; units per chunk; first item of its group's prefix
    int gblocks, grow, pad[2];        // row blocks of its group, and the sequence's first row in them
};
struct SharedNotes {
    SharedNote* note;         // [n]
    int32_t* block;           // [n + 1] row blocks of the sequences ahead of each one's
};

// The parts of up to 64 sequences and groups: a lane's sequence and a lane's group.
struct Parts {
    int tok, n, len, start, group;            // sequence: first token, tokens, length, first key of its own, group
    int gtok, gn, gkeys, gseq;                // group: first token, tokens, P (0: nobody reaches behind it), a sequence that shares
    int blocks, units, gblocks, gunits, c;    // row blocks and units of either; units per chunk
    __device__ __forceinline__ int items() const { return blocks * ceil_div(units, c, 1.f / (float)c); }
    __device__ __forceinline__ int gitems() const { return gblocks * ceil_div(gunits, c, 1.f / (float)c); }
};
__device__ __forceinline__ Parts parts64(const SharedParams& p) {
    const int lane = threadIdx.x & 63, n = p.s.n, groups = p.groups, cap = p.c.max_pages << p.c.shift;
    Parts q;
    q.len = lane < n ? max(p.s.lens[lane], 0) : 0;
    int P = lane < groups ? p.prefix[lane] : 0, gend = lane < groups && p.cu_groups ? p.cu_groups[lane + 1] : 0;
    int at = 0, end;
    span64(p.s, 0, at, q.tok, end);
    q.n = end - q.tok;
    gend = p.cu_groups ? scan_max(lane < groups ? min(max(gend, 0), n) : 0) : n;
    const int gbeg = p.cu_groups ? lane_before(gend, 0) : lane == 0 ? 0 : n;
    P = min(max(P, 0), cap) >> p.c.shift << p.c.shift;
    q.group = 0;
    for (int g = 0; g < groups; ++g) q.group += __builtin_amdgcn_readlane(gend, g) <= lane;
    const int mine = __shfl(P, min(q.group, groups - 1), 64);
    const bool shares = q.group < groups && mine > 0 && q.n > 0 && q.len - q.n >= mine;
    q.start = shares ? mine : 0;
    q.gseq = -1;
    for (int g = 0; g < groups; ++g) {
        const uint64_t any = __builtin_amdgcn_ballot_w64(shares && q.group == g);
        if (lane == g && any) q.gseq = __builtin_ctzll(any);
    }
    const int first = __shfl(end, max(gbeg - 1, 0), 64), last = __shfl(end, max(gend - 1, 0), 64);   // (a sequence's tokens end where the next one's begin)
    q.gtok = gbeg > 0 ? first : 0;
    q.gn = gend > 0 ? last - q.gtok : 0;
    q.gkeys = q.gseq >= 0 ? P : 0;
    q.blocks = (q.n * p.G + p.rbt - 1) / p.rbt;
    q.units = max((min(q.len, cap) - q.start + UNIT - 1) / UNIT, 1);
    q.gblocks = q.gseq >= 0 ? (q.gn * p.G + p.rbp - 1) / p.rbp : 0;
    q.gunits = (q.gkeys + UNIT - 1) / UNIT;
    const double all = lane64(scan64((double)q.blocks * q.units + (double)q.gblocks * q.gunits), 63);
    q.c = __builtin_amdgcn_readfirstlane(chunk_units(all, p.round));
    return q;
}

// The last index i of [0, n) with first[i] <= w (`first` nondecreasing, its next entry past w), by a whole wave; -1 where
// w is past the last.
__device__ __forceinline__ int part_of(const int32_t* first, int n, int w) {
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = n;
    for (;;) {
        const int step = (hi - lo + 63) / 64, at = min(lo + (lane + 1) * step, hi);
        const uint64_t past = __builtin_amdgcn_ballot_w64(at > lo + lane * step && first[at] > w);
        if (!past) return -1;
        lo += __builtin_ctzll(past) * step;
        hi = min(lo + step, hi);
        if (step <= 1) return lo;
    }
}

template <int RB> __device__ __forceinline__ bool find_item(const SharedParams& p, int w, Item& it) {
    int s, a, b, c;
    if (p.part) {
        s = part_of(p.first, p.parts, w);
        if (s < 0) return false;
        const int* x = reinterpret_cast<const int*>(p.part + s);
        it.tok = tab(x, 0);
        it.n = tab(x, 1);
        a = tab(x, 2);
        b = tab(x, 3);
        it.first = tab(p.first, s);
        c = tab(p.chunk, 0);
    } else {
        const Parts q = parts64(p);
        const int x = p.of_prefix ? q.gitems() : q.items(), y = scan_add(x);
        const uint64_t past = __builtin_amdgcn_ballot_w64(y > w);
        if (!past) return false;
        s = __builtin_ctzll(past);
        auto of = [s](int x) { return __builtin_amdgcn_readlane(x, s); };
        it.tok = of(p.of_prefix ? q.gtok : q.tok);
        it.n = of(p.of_prefix ? q.gn : q.n);
        a = of(p.of_prefix ? q.gkeys : q.len);
        b = of(p.of_prefix ? q.gseq : q.start);
        it.first = of(y - x);
        c = q.c;
    }
    it.nrb = (it.n * p.G + RB - 1) / RB;
    const int r = w - it.first;
    it.chunk = r / it.nrb;
    const int z = r - it.chunk * it.nrb;
    it.rb = it.chunk % 2 ? z : it.nrb - 1 - z;   // see item_of
    if (p.of_prefix) {
        it.s = b;
        it.len = a + it.n + AKB;   // (every row sees every key, and those of the last block behind them)
        it.start = 0;
        it.end = a;
    } else {
        it.s = s;
        it.len = a;
        it.start = b;
        it.end = block_end<RB>(p, it.n, a, it.rb);
    }
    cut_keys(it, it.end - it.start, c);
    it.direct = !p.of_prefix && it.start == 0 && it.chunks == 1;
    return true;
}

// The notes of up to 64 sequences, by a wave.
__device__ __forceinline__ void write_notes(const SharedParams& p, const SharedNotes& to) {
    const int lane = threadIdx.x & 63;
    const Parts q = parts64(p);
    const int b = scan_add(q.blocks), x = q.items(), y = scan_add(x), gx = q.gitems(), gy = scan_add(gx), g = min(q.group, 63);
    const int gfirst = __shfl(gy - gx, g, 64), gblocks = __shfl(q.gblocks, g, 64), gtok = __shfl(q.gtok, g, 64);
    if (lane < p.s.n) {   // (three vectors: as one struct it went through scratch memory)
        int4* at = reinterpret_cast<int4*>(to.note + lane);
        at[0] = int4{q.tok, q.n, q.len, q.start};
        at[1] = int4{y - x, b - q.blocks, q.c, gfirst};
        at[2] = int4{gblocks, (q.tok - gtok) * p.G, 0, 0};
        to.block[lane + 1] = b;
    }
    if (lane == 0) to.block[0] = 0;
}

// ------------------------------------------------------------------ k_attn_shared
// FORM: both parts by blocks of 16 rows; the prefixes by blocks of 128; both by blocks of 128.
// One launch, so that the sequences' keys, which memory bounds, are read beside the prefixes' products: two launches one after the
// other took 21.5 and 35.4 us, this one 45, for 64 sequences behind 8192 tokens with 64 to 2000 of their own (179 MB, 4.0 TB/s;
// 16 heads over 8, as below).  A prefix is bound by the tile's steps, not by memory: 65536 tokens in e4m3 under 48 sequences, 151 MB,
// 74 us.  (With weights in one bf16 number 62; 2.85 us for two workgroups' blocks of 64 keys on a CU, of which products, exponentials,
// loads and conversions were 1.3 to 8 of the 61 us each when left out.)  Tried there, with those weights, without gain: blocks of 32
// keys with loads three and four ahead (70 against 64), tiles shared out over the waves, all of a block's LDS reads ahead of its
// products (spills), an item's head tied to an XCD.
template <int DH, typename CT, int FORM>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_attn_shared(SharedParams g, SharedParams t, int prefix_wgs, SharedNotes notes) {
    if (blockIdx.x == 0 && threadIdx.x < 64 && !g.part) write_notes(t, notes);
    const bool prefix = (int)blockIdx.x < prefix_wgs;
    const int wg = (int)blockIdx.x - (prefix ? 0 : prefix_wgs);
    SharedParams p = t;   // (field by field: a choice between the two went through scratch memory)
    if (prefix) {
        p.of_prefix = true;
        p.part = g.part;
        p.first = g.first;
        p.parts = g.parts;
        p.pml = g.pml;
        p.po = g.po;
    }
    if constexpr (FORM == 0) {
        __shared__ __align__(16) float out[NT / 64][16 * ROWS_PITCH<DH>];
        __shared__ float2 ml[NT / 64][16];
        __shared__ int redo;
        attn_rows<DH, CT>(p, wg, [&](int z) -> float* { return out[z]; }, ml, redo);
    } else {
        __shared__ __align__(16) bf16_t k_even[AKB * DH], v_even[AKB * DH], k_odd[AKB * DH], v_odd[AKB * DH];
        __shared__ int odd;
        if (FORM == 2 || prefix) {
            attn_tile<DH, CT, true>(p, wg, k_even, v_even, k_odd, v_odd, odd);
        } else {
            static_assert(16 * ROWS_PITCH<DH> * sizeof(float) <= sizeof k_even, "a wave's sums in a ring slot");
            __shared__ float2 ml[NT / 64][16];
            auto outs = [&](int z) { return reinterpret_cast<float*>(z == 0 ? k_even : z == 1 ? v_even : z == 2 ? k_odd : v_odd); };
            attn_rows<DH, CT>(p, wg, outs, ml, odd);
        }
    }
}

// ------------------------------------------------------------------ k_shared_setup
// One workgroup works out the parts of more than 64 sequences, for all.  Bound by latency: 3 us more a call (see above), since the
// lengths come from the device and every later wave waits for them.
constexpr int SHARED_SEQS = 2048;   // sequences of a call

struct SharedSetup {
    SharedParams p;
    int4* grp;                // [groups], [n]: the parts
    int4* seq;
    int32_t* first_p;         // [groups + 1], [n + 1]: items
    int32_t* first_t;
    int32_t* chunk;
    SharedNotes notes;
};

// The first index i of [0, n) with ends[i] > x (ends nondecreasing), n where there is none.
__device__ __forceinline__ int first_past(const int32_t* ends, int n, int x) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (ends[mid] > x) hi = mid; else lo = mid + 1;
    }
    return lo;
}

// Inclusive scans over the workgroup (of NW waves) of values of 0 or more; `all`: over all threads.
template <int NW, typename F> __device__ __forceinline__ int wg_scan(int x, F f, int* red, int& all) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    x = wave_scan(x, f);
    __syncthreads();   // (red is free)
    if (lane == 63) red[wave] = x;
    __syncthreads();
    int y = lane < NW ? red[lane] : 0;
    y = wave_scan(y, f);
    all = __builtin_amdgcn_readlane(y, NW - 1);
    const int before = __shfl(y, max(wave - 1, 0), 64);
    return wave > 0 ? f(x, before) : x;
}

__global__ __launch_bounds__(NT) void k_shared_setup(SharedSetup u) {
    const SharedParams& p = u.p;
    constexpr int NW = NT / 64;
    __shared__ int tok[SHARED_SEQS + 1], len[SHARED_SEQS], start[SHARED_SEQS], group[SHARED_SEQS];
    __shared__ int gend[SHARED_SEQS], gkeys[SHARED_SEQS], gseq[SHARED_SEQS], gfirst[SHARED_SEQS];
    __shared__ int2 work[2 * SHARED_SEQS];   // row blocks and units of the groups, then of the sequences
    __shared__ int red[NW];
    const int tid = threadIdx.x, lane = tid & 63, n = p.s.n, groups = p.groups, cap = p.c.max_pages << p.c.shift;
    auto most = [](int a, int b) { return max(a, b); };
    auto sum = [](int a, int b) { return a + b; };
    // groups: their sequences end at gend; whole pages of their prefixes (offsets outside the contract are clamped as in span64).
    // Sequences: tokens and lengths.  All of the first NT's values are asked for before any is used.
    int carry_g = 0, carry = 0, all;
    if (tid == 0) tok[0] = 0;
    for (int base = 0; base < max(n, groups); base += NT) {
        const int i = base + tid;
        const int L = i < n ? p.s.lens[i] : 0, P = i < groups ? p.prefix[i] : 0;
        int e = i < n && p.s.cu ? p.s.cu[i + 1] : 0, g = i < groups && p.cu_groups ? p.cu_groups[i + 1] : 0;
        if (p.cu_groups) {
            g = max(wg_scan<NW>(min(max(g, 0), n), most, red, all), carry_g);
            carry_g = max(carry_g, all);
        } else {
            g = n;
        }
        if (p.s.cu) {
            e = max(wg_scan<NW>(min(max(e, 0), p.s.T), most, red, all), carry);
            carry = max(carry, all);
        } else {
            e = (i + 1) * p.s.T;
        }
        if (i < groups) {
            gend[i] = g;
            gkeys[i] = min(max(P, 0), cap) >> p.c.shift << p.c.shift;
            gseq[i] = 1 << 30;
        }
        if (i < n) {
            len[i] = max(L, 0);
            tok[i + 1] = e;
        }
    }
    __syncthreads();
    for (int i = tid; i < n; i += NT) {
        const int g = first_past(gend, groups, i);
        const int m = tok[i + 1] - tok[i], P = g < groups ? gkeys[g] : 0;
        const bool shares = P > 0 && m > 0 && len[i] - m >= P;
        if (shares) atomicMin(&gseq[g], i);
        start[i] = shares ? P : 0;
        group[i] = g;
        u.seq[i] = int4{tok[i], m, len[i], start[i]};
        work[groups + i] = int2{(m * p.G + p.rbt - 1) / p.rbt, max((min(len[i], cap) - start[i] + UNIT - 1) / UNIT, 1)};
    }
    __syncthreads();
    for (int g = tid; g < groups; g += NT) {
        const int from = g > 0 ? gend[g - 1] : 0, m = tok[gend[g]] - tok[from];
        const bool any = gseq[g] < n;
        u.grp[g] = int4{tok[from], m, any ? gkeys[g] : 0, any ? gseq[g] : 0};
        work[g] = int2{any ? (m * p.G + p.rbp - 1) / p.rbp : 0, (gkeys[g] + UNIT - 1) / UNIT};
    }
    __syncthreads();
    double total = 0.;
    for (int i = lane; i < groups + n; i += 64) total += (double)work[i].x * work[i].y;
    const int c = chunk_units(lane64(scan64(total), 63), p.round);
    const float rc = 1.f / (float)c;
    if (tid == 0) {
        u.chunk[0] = c;
        u.first_p[0] = u.first_t[0] = u.notes.block[0] = 0;
    }
    // items, and row blocks of the sequences
    carry = 0;
    for (int base = 0; base < groups; base += NT) {
        const int g = base + tid, x = g < groups ? work[g].x * ceil_div(work[g].y, c, rc) : 0;
        const int y = groups > 1 ? wg_scan<NW>(x, sum, red, all) : x;
        if (g < groups) {
            gfirst[g] = carry + y - x;
            u.first_p[g + 1] = carry + y;
        }
        if (groups > 1) carry += all;
    }
    __syncthreads();
    int carry_b = 0;
    carry = 0;
    for (int base = 0; base < n; base += NT) {
        const int i = base + tid, b = i < n ? work[groups + i].x : 0, x = i < n ? b * ceil_div(work[groups + i].y, c, rc) : 0;
        const int y = carry + wg_scan<NW>(x, sum, red, all);
        carry += all;
        int z = (i + 1) * b;   // (a dense step's sequences have as many row blocks each)
        if (p.s.cu) {
            z = carry_b + wg_scan<NW>(b, sum, red, all);
            carry_b += all;
        }
        if (i < n) {
            u.first_t[i + 1] = y;
            u.notes.block[i + 1] = z;
            const int g = start[i] > 0 ? group[i] : -1;
            u.notes.note[i] = {tok[i], tok[i + 1] - tok[i], len[i], start[i], y - x, z - b, c, g >= 0 ? gfirst[g] : 0,
                               g >= 0 ? work[g].x : 0, g >= 0 ? (tok[i] - tok[g > 0 ? gend[g - 1] : 0]) * p.G : 0, {0, 0}};
        }
    }
}

// ------------------------------------------------------------------ k_shared_join
// One workgroup per row (or, WAVE, one wave: blockIdx.y holds NT / 64 of them) of a row block of the sequences' own keys and
// key/value head: the block's chunks, then those of the prefix, as k_attn_join adds them up.  Bound by latency: the block's
// sequence, its numbers, the partial sums.  Rows that a workgroup each has resident at once are best split over its waves where
// a long prefix left each many partial sums (32, 64 and 128 rows behind 30000 tokens: 21.1, 21.9 and 21.3 us a call against 38.9,
// 31.2 and 30.8 with a wave a row; behind 1000 alike); more rows are best a wave each (4608 rows: 7.5 us, with a workgroup 12.2).
// With twice the loads of a wave at once, 16 a lane, those take 8.6.
struct SharedJoin {
    SharedParams t;           // the sequences' own keys, and their partial sums
    SharedParams g;           // the groups' prefixes
    SharedNotes notes;
    int each;                 // row blocks of a dense step's sequence, or 0
};

template <int DH, bool WAVE>
__global__ __launch_bounds__(NT) void k_shared_join(SharedJoin p) {
    constexpr int LPR = DH / 4, SUB = 64 / LPR, NW = WAVE ? 1 : NT / 64;   // lanes per row; chunks that a wave's load takes at once; waves a row
    __shared__ __align__(16) float red[NW][DH];
    const int lane = threadIdx.x & 63, at = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = WAVE ? 0 : at;
    const int b = div_by(blockIdx.x, p.t.by_hkv), hk = (int)blockIdx.x - b * p.t.HKV, c4 = 4 * (lane % LPR), HKV = p.t.HKV, G = p.t.G;
    const int s = p.each ? b / p.each : part_of(p.notes.block, p.t.s.n, b);
    if (s < 0) return;
    const int* x = reinterpret_cast<const int*>(p.notes.note + s);
    Item it, gr;
    it.tok = tab(x, 0);
    it.n = tab(x, 1);
    it.len = tab(x, 2);
    it.start = tab(x, 3);
    it.first = tab(x, 4);
    it.rb = b - tab(x, 5);
    const int c = tab(x, 6), row0 = tab(x, 9);
    gr.first = tab(x, 7);
    gr.nrb = tab(x, 8);
    it.nrb = (it.n * G + p.t.rbt - 1) / p.t.rbt;
    it.end = p.t.rbt == 16 ? block_end<16>(p.t, it.n, it.len, it.rb) : block_end<AQ>(p.t, it.n, it.len, it.rb);
    cut_keys(it, it.end - it.start, c);
    if (it.start == 0 && it.chunks == 1) return;
    const int r = WAVE ? (int)blockIdx.y * (NT / 64) + at : (int)blockIdx.y, rr = it.rb * p.t.rbt + r;
    if (r >= p.t.rbt || rr >= it.n * G) return;
    gr.chunks = 0;
    const int row = row0 + rr;   // of the group
    gr.rb = row / p.t.rbp;
    const int rg = row - gr.rb * p.t.rbp;
    if (it.start > 0) cut_keys(gr, it.start, c);
    const int own = it.chunks, chunks = own + gr.chunks;
    auto slot = [&](int j) {   // in the group's partial sums from `own` on
        return j < own ? ((long)item_of(it, j) * HKV + hk) * p.t.rbt + r : ((long)item_of(gr, j - own) * HKV + hk) * p.t.rbp + rg;
    };
    constexpr int STEP = WAVE ? 8 * SUB : 64, EACH = STEP / (NW * SUB);   // chunks at a time, and their loads of a wave, all sent off first
    const int mine = wave * SUB + lane / LPR;
    float M = LOWEST, sum = 0.f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    for (int j0 = 0; j0 < chunks; j0 += STEP) {
        floatx4 y[EACH];
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const int j = j0 + k * NW * SUB + mine;
            y[k] = floatx4{0.f, 0.f, 0.f, 0.f};
            if (j < chunks) y[k] = f4((j < own ? p.t.po : p.g.po) + slot(j) * DH + c4);
        }
        float2 ml = {LOWEST, 0.f};   // of chunk j0 + lane
        if (lane < STEP && j0 + lane < chunks) ml = (j0 + lane < own ? p.t.pml : p.g.pml)[slot(j0 + lane)];
        float top = fmaxf(M, ml.x);
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
        const float a = __builtin_amdgcn_exp2f(M - top), w = __builtin_amdgcn_exp2f(ml.x - top);
        sum = sum * a + w * ml.y;
        o *= a;
        M = top;
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const float z = __shfl(w, k * NW * SUB + mine, 64);
            if (j0 + k * NW * SUB + mine < chunks) o += z * y[k];
        }
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) sum += __shfl_xor(sum, off, 64);   // (in every wave)
#pragma unroll
    for (int off = LPR; off < 64; off <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], off, 64);
    if constexpr (!WAVE) {
        if (lane < LPR) *reinterpret_cast<floatx4*>(&red[wave][c4]) = o;
        __syncthreads();
        o = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int z = 0; z < NW; ++z) o += f4(&red[z][c4]);
    }
    if (wave != 0 || lane >= LPR) return;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const int i = div_by(rr, p.t.by_g);
    bf16_t* dst = p.t.o + ((long)(it.tok + i) * p.t.H + hk * G + rr - i * G) * DH + c4;
    *reinterpret_cast<bf16x4*>(dst) = __builtin_convertvector(o * inv, bf16x4);
}
