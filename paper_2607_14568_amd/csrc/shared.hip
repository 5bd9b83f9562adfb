// Paged attention of a batch whose sequences share long prefixes (included by gdn.hip, behind paged.hip, whose kernels it runs).
//
// The sequences of a group hold the same first P tokens in the same pages.  With softmax weights relative to any reference,
// a row's output over all its keys is the weighted mean of those over the prefix and over what is behind it:
//   m = max(m1, m2),  l = l1 2^(m1 - m) + l2 2^(m2 - m),  o = (o1 2^(m1 - m) + o2 2^(m2 - m)) / l.
// The rows of all the group's new tokens attend the prefix together (each sees all of it, so no key is masked), which reads
// it once for the group, and every sequence's rows attend its own keys behind it.  So one call takes
//   k_shared_setup   the parts: groups and sequences with their keys, chunks and items, from the lengths on the device
//   k_attn_rows or k_attn_tile, twice: over the groups' prefixes and over the sequences' own keys
//   k_shared_join    every row's partial sums added up in order
// A sequence that does not reach behind its group's prefix (a finished one, one that does not belong) takes no part in it and
// attends all its keys by itself.

struct SharedParams : PagedParams {
    const int4* part;         // groups {first token, tokens, P, a sequence that shares}, or sequences {first token, tokens, length, start}
    const int32_t* first;     // [parts + 1] items of one key/value head ahead of each part's
    const int32_t* chunk;     // units per chunk
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

// ------------------------------------------------------------------ k_shared_setup
// One workgroup.  A part's keys are cut into chunks of c units so that all items are resident at once where that can be:
// c0 = ceil(all row blocks' units / round) at least, and of the next 31 c that grow by a sixteenth the first with at most
// `round` items; where none has, c0 itself, with at most round + (row blocks) items (ceil(u / c) < u / c + 1).
constexpr int SHARED_SEQS = 2048, NSU = 1024;   // sequences of a call; threads

struct SharedSetup {
    StepSeqs s;
    const int32_t* prefix;    // [groups] tokens that a group's sequences share
    const int32_t* cu_groups; // [groups + 1] offsets of the groups among the sequences; null: one group
    int groups, G, shift, cap;
    int rbp, rbt, round_p, round_t;   // rows per block, and items at once, of the prefixes and of the sequences' own keys
    int least_p, least_t;             // units of a chunk at least
    int4* grp;                // [groups], [n]: the parts
    int4* seq;
    int32_t* group_of;        // [n]: group whose prefix a sequence attends, or -1
    int32_t* first_p;         // [groups + 1], [n + 1]: items
    int32_t* first_t;
    int32_t* block_t;         // [n + 1]: row blocks of the sequences
    int32_t* chunk;           // of the prefixes, of the own keys
};

// Inclusive scan over the workgroup of values of 0 or more; `all`: over all threads.
template <typename F> __device__ __forceinline__ int wg_scan(int x, F f, int* red, int& all) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    x = wave_scan(x, f);
    __syncthreads();   // (red is free)
    if (lane == 63) red[wave] = x;
    __syncthreads();
    int y = lane < NSU / 64 ? red[lane] : 0;
    y = wave_scan(y, f);
    all = __builtin_amdgcn_readlane(y, NSU / 64 - 1);
    const int before = __shfl(y, max(wave - 1, 0), 64);
    return wave > 0 ? f(x, before) : x;
}

// Units per chunk of parts with blocks[i] row blocks of units[i] units each (see above).
__device__ __forceinline__ int chunk_units(const int* blocks, const int* units, int n, int round, int least, int* red) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, tid = threadIdx.x;
    float total = 0.f;
    for (int i = lane; i < n; i += 64) total += (float)blocks[i] * (float)units[i];
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) total += __shfl_xor(total, off, 64);
    const int c0 = max((int)min(ceilf(total * (1.f + 0x1p-17f) / (float)round), 0x1p23f), least);   // (sums of 2048 floats: 2^-18 off at most)
    __syncthreads();
    for (int k = wave; k < 32; k += NSU / 64) {
        const int c = c0 + (c0 * k + 15) / 16;
        const float rc = 1.f / (float)c;
        int sum = 0;
        for (int i = lane; i < n; i += 64) sum = (int)min((long)blocks[i] * ceil_div(units[i], c, rc) + sum, 1L << 24);
        sum = last_lane(scan_add(sum));
        if (lane == 0) red[k] = sum;
    }
    __syncthreads();
    const uint64_t fits = __builtin_amdgcn_ballot_w64(lane < 32 && red[lane & 31] <= round);
    const int k = fits ? __builtin_ctzll(fits) : 0;
    __syncthreads();
    (void)tid;
    return c0 + (c0 * k + 15) / 16;
}

__global__ __launch_bounds__(NSU) void k_shared_setup(SharedSetup p) {
    __shared__ int tok[SHARED_SEQS + 1], len[SHARED_SEQS], start[SHARED_SEQS], units[SHARED_SEQS], blocks[SHARED_SEQS];
    __shared__ int gend[SHARED_SEQS], gkeys[SHARED_SEQS], gseq[SHARED_SEQS];
    __shared__ int red[32];
    const int tid = threadIdx.x, n = p.s.n;
    auto most = [](int a, int b) { return max(a, b); };
    auto sum = [](int a, int b) { return a + b; };
    // sequences: tokens (offsets outside the contract are clamped as in span64) and lengths
    int carry = 0, all;
    if (tid == 0) tok[0] = 0;
    for (int base = 0; base < n; base += NSU) {
        const int i = base + tid;
        if (i < n) len[i] = max(p.s.lens[i], 0);
        if (p.s.cu) {
            const int e = max(wg_scan(i < n ? min(max(p.s.cu[i + 1], 0), p.s.T) : 0, most, red, all), carry);
            carry = max(carry, all);
            if (i < n) tok[i + 1] = e;
        } else if (i < n) {
            tok[i + 1] = (i + 1) * p.s.T;
        }
    }
    // groups: their sequences end at gend; whole pages of their prefixes
    carry = 0;
    for (int base = 0; base < p.groups; base += NSU) {
        const int g = base + tid;
        int e = g < p.groups ? (p.cu_groups ? min(max(p.cu_groups[g + 1], 0), n) : n) : 0;
        e = max(wg_scan(e, most, red, all), carry);
        carry = max(carry, all);
        if (g < p.groups) {
            gend[g] = e;
            gkeys[g] = min(max(p.prefix[g], 0), p.cap) >> p.shift << p.shift;
            gseq[g] = 1 << 30;
        }
    }
    __syncthreads();
    for (int i = tid; i < n; i += NSU) {
        int lo = 0, hi = p.groups;   // the first group that ends behind i
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (gend[mid] > i) hi = mid; else lo = mid + 1;
        }
        const int m = tok[i + 1] - tok[i], P = lo < p.groups ? gkeys[lo] : 0;
        const bool shares = P > 0 && m > 0 && len[i] - m >= P;
        if (shares) atomicMin(&gseq[lo], i);
        start[i] = shares ? P : 0;
        p.group_of[i] = shares ? lo : -1;
        p.seq[i] = int4{tok[i], m, len[i], start[i]};
    }
    __syncthreads();
    // items of the prefixes
    for (int g = tid; g < p.groups; g += NSU) {
        const int from = g > 0 ? gend[g - 1] : 0, m = tok[gend[g]] - tok[from];
        const bool any = gseq[g] < n;
        p.grp[g] = int4{tok[from], m, any ? gkeys[g] : 0, any ? gseq[g] : 0};
        blocks[g] = any ? (m * p.G + p.rbp - 1) / p.rbp : 0;
        units[g] = (gkeys[g] + UNIT - 1) / UNIT;
    }
    __syncthreads();
    const int cp = chunk_units(blocks, units, p.groups, p.round_p, p.least_p, red);
    carry = 0;
    if (tid == 0) {
        p.chunk[0] = cp;
        p.first_p[0] = 0;
    }
    for (int base = 0; base < p.groups; base += NSU) {
        const int g = base + tid, x = g < p.groups ? blocks[g] * ((units[g] + cp - 1) / cp) : 0, y = wg_scan(x, sum, red, all);
        if (g < p.groups) p.first_p[g + 1] = carry + y;
        carry += all;
    }
    __syncthreads();
    // ... and of the sequences' own keys
    for (int i = tid; i < n; i += NSU) {
        blocks[i] = ((tok[i + 1] - tok[i]) * p.G + p.rbt - 1) / p.rbt;
        units[i] = max((min(len[i], p.cap) - start[i] + UNIT - 1) / UNIT, 1);
    }
    __syncthreads();
    const int ct = chunk_units(blocks, units, n, p.round_t, p.least_t, red);
    int carry_b = 0;
    carry = 0;
    if (tid == 0) {
        p.chunk[1] = ct;
        p.first_t[0] = p.block_t[0] = 0;
    }
    for (int base = 0; base < n; base += NSU) {
        const int i = base + tid, b = i < n ? blocks[i] : 0, x = i < n ? b * ((units[i] + ct - 1) / ct) : 0;
        const int y = wg_scan(x, sum, red, all);
        if (i < n) p.first_t[i + 1] = carry + y;
        carry += all;
        const int z = wg_scan(b, sum, red, all);
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
