// Paged attention of a batch whose sequences share long prefixes (included by gdn.hip, behind paged.hip, whose kernels it runs).
//
// The sequences of a group hold the same first P tokens in the same pages.  With softmax weights relative to any reference,
// a row's output over all its keys is the weighted mean of those over the prefix and over what is behind it:
//   m = max(m1, m2),  l = l1 2^(m1 - m) + l2 2^(m2 - m),  o = (o1 2^(m1 - m) + o2 2^(m2 - m)) / l.
// The rows of all the group's new tokens attend the prefix together (each sees all of it, so no key is masked), which reads
// it once for the group, and every sequence's rows attend its own keys behind it.  So one call takes
//   k_shared_setup   the parts: groups and sequences with their keys, chunks and items, from the lengths on the device
//   k_attn_shared    the items, of the groups' prefixes (first in the grid) and of the sequences' own keys, by the workgroups of
//                    k_attn_rows and k_attn_tile
//   k_shared_join    every row's partial sums added up in order
// A sequence that does not reach behind its group's prefix (a finished one, one that does not belong) takes no part in it and
// attends all its keys by itself.

struct SharedParams : PagedParams {
    const int4* part;         // groups {first token, tokens, P, a sequence that shares}, or sequences {first token, tokens, length, start}
    const int32_t* first;     // [parts + 1] items of one key/value head ahead of each part's
    const int32_t* chunk;     // units per chunk (one word)
    int parts;
    bool prefix;
};

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
    const int s = part_of(p.first, p.parts, w);
    if (s < 0) return false;
    const int* x = reinterpret_cast<const int*>(p.part + s);
    it.tok = tab(x, 0);
    it.n = tab(x, 1);
    const int a = tab(x, 2), b = tab(x, 3);
    it.nrb = (it.n * p.G + RB - 1) / RB;
    it.first = tab(p.first, s);
    const int r = w - it.first;
    it.chunk = r / it.nrb;
    const int z = r - it.chunk * it.nrb;
    it.rb = it.chunk % 2 ? z : it.nrb - 1 - z;   // see item_of
    if (p.prefix) {
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
    cut_keys(it, it.end - it.start, tab(p.chunk, 0));
    it.direct = !p.prefix && it.start == 0 && it.chunks == 1;
    return true;
}

// ------------------------------------------------------------------ k_attn_shared
// FORM: both parts by blocks of 16 rows; the prefixes by blocks of 128; both by blocks of 128.
template <int DH, typename CT, int FORM>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_attn_shared(SharedParams g, SharedParams t, int prefix_wgs) {
    const bool prefix = (int)blockIdx.x < prefix_wgs;
    const int wg = (int)blockIdx.x - (prefix ? 0 : prefix_wgs);
    const SharedParams& p = prefix ? g : t;
    if constexpr (FORM == 0) {
        __shared__ __align__(16) float out[NT / 64][16 * ROWS_PITCH<DH>];
        __shared__ float2 ml[NT / 64][16];
        __shared__ int redo;
        attn_rows<DH, CT>(p, wg, [&](int z) -> float* { return out[z]; }, ml, redo);
    } else {
        __shared__ __align__(16) bf16_t k_even[AKB * DH], v_even[AKB * DH], k_odd[AKB * DH], v_odd[AKB * DH];
        __shared__ int odd;
        if (FORM == 2 || prefix) {
            attn_tile<DH, CT>(p, wg, k_even, v_even, k_odd, v_odd, odd);
        } else {
            static_assert(16 * ROWS_PITCH<DH> * sizeof(float) <= sizeof k_even, "a wave's sums in a ring slot");
            __shared__ float2 ml[NT / 64][16];
            auto outs = [&](int z) { return reinterpret_cast<float*>(z == 0 ? k_even : z == 1 ? v_even : z == 2 ? k_odd : v_odd); };
            attn_rows<DH, CT>(p, wg, outs, ml, odd);
        }
    }
}

// ------------------------------------------------------------------ k_shared_setup
// One workgroup.  All parts' keys are cut into chunks of c units, so that all items are resident at once where that can be:
// c0 = ceil(all row blocks' units / round) at least, and of the next 31 c that grow by a sixteenth the first with at most
// `round` items; where none has, c0 itself, with at most round + (row blocks) items (ceil(u / c) < u / c + 1).
// Bound by latency.
constexpr int SHARED_SEQS = 2048;   // sequences of a call

struct SharedSetup {
    StepSeqs s;
    const int32_t* prefix;    // [groups] tokens that a group's sequences share
    const int32_t* cu_groups; // [groups + 1] offsets of the groups among the sequences; null: one group
    int groups, G, shift, cap;
    int rbp, rbt;             // rows per block of the prefixes and of the sequences' own keys
    int round, least;         // items at once (of both); units of a chunk at least
    int4* grp;                // [groups], [n]: the parts
    int4* seq;
    int32_t* group_of;        // [n]: group whose prefix a sequence attends, or -1
    int32_t* first_p;         // [groups + 1], [n + 1]: items
    int32_t* first_t;
    int32_t* block_t;         // [n + 1]: row blocks of the sequences
    int32_t* chunk;
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

__global__ __launch_bounds__(NT) void k_shared_setup(SharedSetup p) {
    constexpr int NW = NT / 64;
    __shared__ int tok[SHARED_SEQS + 1], len[SHARED_SEQS];
    __shared__ int gend[SHARED_SEQS], gkeys[SHARED_SEQS], gseq[SHARED_SEQS];
    __shared__ int blocks[2 * SHARED_SEQS], units[2 * SHARED_SEQS];   // of the groups, then of the sequences
    __shared__ int red[32];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = p.s.n, groups = p.groups;
    auto most = [](int a, int b) { return max(a, b); };
    auto sum = [](int a, int b) { return a + b; };
    int carry = 0, all;
    if (tid == 0) tok[0] = 0;
    // groups: their sequences end at gend; whole pages of their prefixes (offsets outside the contract are clamped as in span64)
    for (int base = 0; base < groups; base += NT) {
        const int g = base + tid;
        int e = n;
        if (g < groups) {
            gkeys[g] = min(max(p.prefix[g], 0), p.cap) >> p.shift << p.shift;
            gseq[g] = 1 << 30;
        }
        if (p.cu_groups) {
            e = max(wg_scan<NW>(g < groups ? min(max(p.cu_groups[g + 1], 0), n) : 0, most, red, all), carry);
            carry = max(carry, all);
        }
        if (g < groups) gend[g] = e;
    }
    // sequences: tokens and lengths
    carry = 0;
    for (int base = 0; base < n; base += NT) {
        const int i = base + tid;
        if (i < n) len[i] = max(p.s.lens[i], 0);
        if (p.s.cu) {
            const int e = max(wg_scan<NW>(i < n ? min(max(p.s.cu[i + 1], 0), p.s.T) : 0, most, red, all), carry);
            carry = max(carry, all);
            if (i < n) tok[i + 1] = e;
        } else if (i < n) {
            tok[i + 1] = (i + 1) * p.s.T;
        }
    }
    __syncthreads();
    for (int i = tid; i < n; i += NT) {
        const int g = first_past(gend, groups, i);
        const int m = tok[i + 1] - tok[i], P = g < groups ? gkeys[g] : 0;
        const bool shares = P > 0 && m > 0 && len[i] - m >= P;
        if (shares) atomicMin(&gseq[g], i);
        const int from = shares ? P : 0;
        p.group_of[i] = shares ? g : -1;
        p.seq[i] = int4{tok[i], m, len[i], from};
        blocks[groups + i] = (m * p.G + p.rbt - 1) / p.rbt;
        units[groups + i] = max((min(len[i], p.cap) - from + UNIT - 1) / UNIT, 1);
    }
    __syncthreads();
    for (int g = tid; g < groups; g += NT) {
        const int from = g > 0 ? gend[g - 1] : 0, m = tok[gend[g]] - tok[from];
        const bool any = gseq[g] < n;
        p.grp[g] = int4{tok[from], m, any ? gkeys[g] : 0, any ? gseq[g] : 0};
        blocks[g] = any ? (m * p.G + p.rbp - 1) / p.rbp : 0;
        units[g] = (gkeys[g] + UNIT - 1) / UNIT;
    }
    __syncthreads();
    // units per chunk
    float total = 0.f;
    for (int i = lane; i < groups + n; i += 64) total += (float)blocks[i] * (float)units[i];
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) total += __shfl_xor(total, off, 64);
    const int c0 = max((int)min(ceilf(total * (1.f + 0x1p-17f) / (float)p.round), 0x1p23f), p.least);   // (sums of 64 floats a lane: 2^-18 off at most)
    for (int k = wave; k < 32; k += NW) {
        const int c = c0 + (c0 * k + 15) / 16;
        const float rc = 1.f / (float)c;
        int x = 0;
        for (int i = lane; i < groups + n; i += 64) x = (int)min((long)blocks[i] * ceil_div(units[i], c, rc) + x, 1L << 24);
        x = last_lane(scan_add(x));
        if (lane == 0) red[k] = x;
    }
    __syncthreads();
    const uint64_t fits = __builtin_amdgcn_ballot_w64(lane < 32 && red[lane & 31] <= p.round);
    const int c = c0 + (c0 * (fits ? __builtin_ctzll(fits) : 0) + 15) / 16;
    const float rc = 1.f / (float)c;
    if (tid == 0) {
        p.chunk[0] = c;
        p.first_p[0] = p.first_t[0] = p.block_t[0] = 0;
    }
    // items, and row blocks of the sequences
    carry = 0;
    for (int base = 0; base < groups; base += NT) {
        const int g = base + tid, y = wg_scan<NW>(g < groups ? blocks[g] * ceil_div(units[g], c, rc) : 0, sum, red, all);
        if (g < groups) p.first_p[g + 1] = carry + y;
        carry += all;
    }
    int carry_b = 0;
    carry = 0;
    for (int base = 0; base < n; base += NT) {
        const int i = base + tid, b = i < n ? blocks[groups + i] : 0;
        const int y = wg_scan<NW>(i < n ? b * ceil_div(units[groups + i], c, rc) : 0, sum, red, all);
        if (i < n) p.first_t[i + 1] = carry + y;
        carry += all;
        const int z = wg_scan<NW>(b, sum, red, all);
        if (i < n) p.block_t[i + 1] = carry_b + z;
        carry_b += all;
    }
}

// ------------------------------------------------------------------ k_shared_join
// One workgroup per row (blockIdx.y) of a row block of the sequences' own keys and key/value head: the block's chunks, then
// those of the prefix, as k_attn_join adds them up.
struct SharedJoin {
    SharedParams t;           // the sequences' own keys, and their partial sums
    SharedParams g;           // the groups' prefixes
    const int32_t* group_of;
    const int32_t* block_t;
    int rbp, rbt;
};

template <int DH>
__global__ __launch_bounds__(NT) void k_shared_join(SharedJoin p) {
    constexpr int LPR = DH / 4, SUB = 64 / LPR, NW = NT / 64;   // lanes per row; chunks that a wave's load takes at once
    __shared__ __align__(16) float red[NW][DH];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = div_by(blockIdx.x, p.t.by_hkv), hk = (int)blockIdx.x - b * p.t.HKV, c4 = 4 * (lane % LPR), HKV = p.t.HKV, G = p.t.G;
    const int s = part_of(p.block_t, p.t.parts, b);
    if (s < 0) return;
    const int* x = reinterpret_cast<const int*>(p.t.part + s);
    Item it;
    it.tok = tab(x, 0);
    it.n = tab(x, 1);
    it.len = tab(x, 2);
    it.start = tab(x, 3);
    it.nrb = (it.n * G + p.rbt - 1) / p.rbt;
    it.first = tab(p.t.first, s);
    it.rb = b - tab(p.block_t, s);
    it.end = p.rbt == 16 ? block_end<16>(p.t, it.n, it.len, it.rb) : block_end<AQ>(p.t, it.n, it.len, it.rb);
    cut_keys(it, it.end - it.start, tab(p.t.chunk, 0));
    if (it.start == 0 && it.chunks == 1) return;
    const int r = blockIdx.y, rr = it.rb * p.rbt + r;
    if (r >= p.rbt || rr >= it.n * G) return;
    Item gr;
    gr.chunks = 0;
    int rg = 0;   // the row in its block of the group
    if (it.start > 0) {
        const int g = tab(p.group_of, s);
        const int* y = reinterpret_cast<const int*>(p.g.part + g);
        const int row = (it.tok - tab(y, 0)) * G + rr;
        gr.n = tab(y, 1);
        gr.end = tab(y, 2);
        gr.nrb = (gr.n * G + p.rbp - 1) / p.rbp;
        gr.rb = row / p.rbp;
        rg = row - gr.rb * p.rbp;
        gr.first = tab(p.g.first, g);
        cut_keys(gr, gr.end, tab(p.g.chunk, 0));
    }
    const int own = it.chunks, chunks = own + gr.chunks;
    auto slot = [&](int j) {   // in the group's partial sums from `own` on
        return j < own ? ((long)item_of(it, j) * HKV + hk) * p.rbt + r : ((long)item_of(gr, j - own) * HKV + hk) * p.rbp + rg;
    };
    constexpr int EACH = 64 / (NW * SUB);   // loads of a wave for 64 chunks, all sent off before the first is used
    const int mine = wave * SUB + lane / LPR;
    float M = LOWEST, sum = 0.f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    for (int j0 = 0; j0 < chunks; j0 += 64) {
        floatx4 y[EACH];
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const int j = j0 + k * NW * SUB + mine;
            y[k] = floatx4{0.f, 0.f, 0.f, 0.f};
            if (j < chunks) y[k] = f4((j < own ? p.t.po : p.g.po) + slot(j) * DH + c4);
        }
        float2 ml = {LOWEST, 0.f};   // of chunk j0 + lane
        if (j0 + lane < chunks) ml = (j0 + lane < own ? p.t.pml : p.g.pml)[slot(j0 + lane)];
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
    if (lane < LPR) *reinterpret_cast<floatx4*>(&red[wave][c4]) = o;
    __syncthreads();
    if (wave != 0 || lane >= LPR) return;
    o = f4(&red[0][c4]);
#pragma unroll
    for (int z = 1; z < NW; ++z) o += f4(&red[z][c4]);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const int i = div_by(rr, p.t.by_g);
    bf16_t* dst = p.t.o + ((long)(it.tok + i) * p.t.H + hk * G + rr - i * G) * DH + c4;
    *reinterpret_cast<bf16x4*>(dst) = __builtin_convertvector(o * inv, bf16x4);
}
