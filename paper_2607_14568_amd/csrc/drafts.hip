// A step of drafted decoding around the layers (included by gdn.hip, behind paged.hip): the pages and slots of a step's
// tokens, the recurrent layers over a few tokens a sequence with the state left at the last kept one, and the verification
// of drafted tokens.

// ------------------------------------------------------------------ k_cache_tables
// Pages of n sequences from and to a pool.  Sequence i holds the pages table[i][0 .. held_i), the first shared_i of them no
// pages of its own; it needs target_i = max(ceil(len_i / page), min(shared_i, held_i)).  Pages behind its target go to the
// pool's end, in order of sequence and entry; then the missing ones, in that order, are the pool's last ones, in theirs (so
// that what one step took and the next gives back lies in the pool as before).
// One workgroup: the sums over the sequences and the pool's end hold everything together, and a step moves a few pages a
// sequence.  Bound by latency: the lengths, the pages given, the pages taken and the slots that need them are loads that
// wait for one another: 3.5 us for 256 sequences' 5 tokens each, with their maps.
struct TablesParams {
    const int32_t* lens;
    const int32_t* new_lens;   // null: rows / n each
    const int32_t* shared;     // or null
    int32_t* table;
    int32_t* held;
    int32_t* free;
    int32_t* n_free;
    int32_t* missing;          // or null
    int32_t* cu;               // or null
    int32_t* positions;        // or null
    int64_t* slots;            // or null
    int n, rows, shift, n_pages, max_pages;
};

// Position, and slot or -1, of a token that is the i-th of m new ones of sequence s, of L tokens.
__device__ __forceinline__ void map_token(const TablesParams& p, int t, int s, int i, int m, int L) {
    const int pos = L - m + i;
    if (p.positions) p.positions[t] = pos;
    if (!p.slots) return;
    int id = -1;
    if (pos >= 0 && pos >> p.shift < p.max_pages) id = p.table[(long)s * p.max_pages + (pos >> p.shift)];
    p.slots[t] = id >= 0 && id < p.n_pages ? ((int64_t)id << p.shift) + (pos & ((1 << p.shift) - 1)) : -1;
}
__device__ __forceinline__ void map_none(const TablesParams& p, int t) {
    if (p.positions) p.positions[t] = 0;
    if (p.slots) p.slots[t] = -1;
}

constexpr int NTA = 1024;   // threads of k_cache_tables, and sequences that it takes at a time

// Inclusive scans over the workgroup of pages given, pages taken and new tokens (running sums held to `rows` < 2^30), in one go.
__device__ __forceinline__ void scan_three(int (&x)[3], int rows, int (*red)[NTA / 64], int (&all)[3]) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    auto sum = [](int a, int b) { return a + b; };
    auto tokens = [rows](int a, int b) { return min(a + b, rows); };
    x[0] = wave_scan(x[0], sum);
    x[1] = wave_scan(x[1], sum);
    x[2] = wave_scan(x[2], tokens);
    __syncthreads();   // (red is free)
    if (lane == 63)
#pragma unroll
        for (int k = 0; k < 3; ++k) red[k][wave] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        int y = lane < NTA / 64 ? red[k][lane] : 0;
        y = k < 2 ? wave_scan(y, sum) : wave_scan(y, tokens);
        all[k] = __builtin_amdgcn_readlane(y, NTA / 64 - 1);
        const int before = __builtin_amdgcn_readlane(y, max(__builtin_amdgcn_readfirstlane(wave) - 1, 0));
        if (wave > 0) x[k] = k < 2 ? sum(x[k], before) : tokens(x[k], before);
    }
}

// maps: the positions and slots too (at most NTA sequences).
__global__ __launch_bounds__(NTA) void k_cache_tables(TablesParams p, int maps) {
    __shared__ int ends[NTA], at[NTA];   // running sums of pages moved, and where they stand in a sequence's row
    __shared__ int cu_ends[NTA], lens[NTA];   // maps: token offsets and lengths
    __shared__ int red[3][NTA / 64];
    const int tid = threadIdx.x, page = 1 << p.shift, rows = p.rows;
    const int have = min(max(p.n_free[0], 0), p.n_pages);
    int held, target, give_end, take_end;   // of sequence base + tid; running sums of its pages given and taken
    // Sums over the sequences [base, base + NTA) (they stay below 2^31: n max_pages does), offsets of their tokens from `token` on.
    int sums[3], token = 0;
    auto load = [&](int base, bool tokens) {
        const int i = base + tid;
        held = target = 0;
        int fresh = 0;
        if (i < p.n) {
            held = min(max(p.held[i], 0), p.max_pages);
            const int len = max(p.lens[i], 0);
            if (p.new_lens && tokens) fresh = min(max(p.new_lens[i], 0), rows);
            target = min((int)(((long)len + page - 1) >> p.shift), p.max_pages);
            if (p.shared) target = max(target, min(p.shared[i], held));
            lens[tid] = len;
        }
        int x[3] = {max(held - target, 0), max(target - held, 0), fresh};
        scan_three(x, rows, red, sums);
        give_end = x[0];
        take_end = x[1];
        if (tokens && i < p.n && p.cu) p.cu[i + 1] = cu_ends[tid] = p.new_lens ? min(token + x[2], rows) : (i + 1) * (rows / p.n);
        token = min(token + sums[2], rows);
    };
    // pages given back
    int given = 0, wanted = 0;
    for (int base = 0; base < p.n; base += NTA) {
        const int m = min(p.n - base, NTA);
        load(base, true);
        wanted += sums[1];
        if (sums[0] > 0) {
            ends[tid] = give_end;
            at[tid] = target - (give_end - max(held - target, 0));
            __syncthreads();
            for (int x = tid; x < sums[0]; x += NTA) {
                const int s = first_past(ends, m, x);
                int32_t* entry = p.table + (long)(base + s) * p.max_pages + at[s] + x;
                const int to = have + given + x;
                if (to < p.n_pages) p.free[to] = *entry;
                *entry = -1;
            }
            given += sums[0];
            __syncthreads();
        }
    }
    if (tid == 0 && p.cu) p.cu[0] = 0;
    const int pool = min(have + given, p.n_pages), got = min(wanted, pool);
    // pages taken
    int taken = 0;
    for (int base = 0; base < p.n; base += NTA) {
        const int i = base + tid, m = min(p.n - base, NTA);
        if (p.n > NTA) load(base, false);
        const int take = max(target - held, 0);
        if (i < p.n) p.held[i] = min(held, target) + min(max(got - taken - (take_end - take), 0), take);
        if (sums[1] > 0) {
            ends[tid] = take_end;
            at[tid] = held - (take_end - take);
            __syncthreads();
            for (int x = tid; x < sums[1]; x += NTA) {
                const int s = first_past(ends, m, x);
                p.table[(long)(base + s) * p.max_pages + at[s] + x] = taken + x < got ? p.free[pool - got + taken + x] : -1;
            }
            taken += sums[1];
            __syncthreads();
        }
    }
    if (tid == 0) {
        p.n_free[0] = pool - got;
        if (p.missing) p.missing[0] = wanted - got;
    }
    if (!maps) return;
    __syncthreads();
    const int T = rows / p.n;
    for (int t = tid; t < rows; t += NTA) {
        if (!p.new_lens) {
            map_token(p, t, t / T, t % T, T, lens[t / T]);
            continue;
        }
        const int s = first_past(cu_ends, p.n, t);
        if (s >= p.n) {
            map_none(p, t);
        } else {
            const int beg = s > 0 ? cu_ends[s - 1] : 0;
            map_token(p, t, s, t - beg, cu_ends[s] - beg, lens[s]);
        }
    }
}

// The positions and slots of many tokens, from the tables and offsets that k_cache_tables left: a thread each, bound by latency.
// Up to 4096 tokens that kernel's workgroup makes them itself, a launch less: 512 of 64 sequences 7.8 us (here 10.1), 2048 of 128
// 9.0 (10.4), 4096 of 8 9.1 (9.1) or of 256 11.2 (10.9), but 8192 of 8 11.5 (9.1) and 32768 25.8 (9.2).
__global__ __launch_bounds__(NT) void k_cache_maps(TablesParams p) {
    const int t = (int)blockIdx.x * NT + threadIdx.x;
    if (t >= p.rows) return;
    if (!p.new_lens) {
        const int T = p.rows / p.n;
        map_token(p, t, t / T, t % T, T, max(p.lens[t / T], 0));
        return;
    }
    const int s = first_past(p.cu + 1, p.n, t);
    if (s >= p.n) {
        map_none(p, t);
        return;
    }
    const int beg = p.cu[s];
    map_token(p, t, s, t - beg, p.cu[s + 1] - beg, max(p.lens[s], 0));
}

// ------------------------------------------------------------------ k_draft_step
// A few tokens of each sequence through a recurrent layer (the recurrence at the head of gdn.hip), the state read once and
// written, where any token is kept, once.  In tiles of TT = 8 tokens, with S the state before the tile:
//   X_t = S k_t,  Y_t = S (scale q_t)                       one product [K; Q] S^T of 16 rows, fp32 matrix instructions
//   u_t = beta_t (v_t - gamma_t X_t - sum_{i<t} c_i (k_t . k_i)),   c_i = u_i decayed from i to t
//   o_t = gamma_t Y_t + sum_{i<=t} c_i (q_t . k_i)          row by row of the state, a row in four lanes alike
//   S'  = gamma_n S + sum_i c_i k_i^T                       c after the n-th token: the next tile's state, or the kept one
// Decays multiply as the tokens pass, so that a gate of 0 (log-decay -inf) is one; nothing is divided.
// A wave holds 16 state rows in registers as accumulators of S^T tiles: lane 16 lg + j has row j's channels 16 b + 4 lg .. + 3,
// which is the layout of a product's operand and result alike, so S enters and leaves them without a move.
// Bound by memory (the state once in, and once out where tokens are kept): 64 sequences, 16 heads of 128, 5 tokens of which 0 to 5
// are kept, 28.5 us (4.6 TB/s; a copy reaches 5.1); the kept ones of 128 sequences' 1 to 9 tokens alone 46.7 us (4.3 TB/s).  What
// the tokens make among themselves (their products, norms, gates) is done while the state is on its way: asked for ahead of
// the tokens it took 33.7 and 55.4 us.  32 rows a wave: 30.6 and 47.6 us.  One sequence, 5.3 us: latency.
constexpr int TT = 8, DROWS = 64;   // tokens of a tile; state rows of a workgroup
struct DraftParams {
    const void* q;            // or null: no outputs
    const void* k;
    const void* v;
    const float* g;
    const float* beta;
    float* S;                 // [n][H][DV][DK]
    void* o;
    const int32_t* keep;      // [n], or null: all
    StepSeqs s;
    int H, HK, G, DV;
    float scale;
    int pre;
};

// The tokens [beg, end) of sequence s, as span64 has them.  Called by a whole wave.
__device__ __forceinline__ void seq_span(const StepSeqs& q, int s, int& beg, int& end) {
    if (!q.cu) {
        beg = s * q.T;
        end = beg + q.T;
        return;
    }
    const int lane = threadIdx.x & 63;
    int m = 0;
    for (int base = 1; base <= s; base += 64) m = max(m, base + lane <= s ? q.cu[base + lane] : 0);
    beg = min(last_lane(scan_max(max(m, 0))), q.T);
    end = min(max(tab(q.cu, s + 1), beg), q.T);
}

// 4 neighbouring values (aligned as one is) in floats
__device__ __forceinline__ floatx4 four(const float* p) {
    typedef floatx4 any __attribute__((aligned(4)));
    return *reinterpret_cast<const any*>(p);
}
__device__ __forceinline__ floatx4 four(const bf16_t* p) {
    typedef short4v any __attribute__((aligned(2)));
    const short4v y = *reinterpret_cast<const any*>(p);
    return floatx4{bf(y[0]), bf(y[1]), bf(y[2]), bf(y[3])};
}

template <typename IO, int DK>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(4))) void k_draft_step(DraftParams p) {
    constexpr int NB = DK / 16, NW = NT / 64, PITCH = DK + 4;
    __shared__ __align__(16) float kq[2 * TT][PITCH];       // keys, then queries, of the tile
    __shared__ __align__(16) float part[NW][2 * TT][TT];    // a wave's share of k_t . k_i and q_t . k_i
    __shared__ __align__(16) float pair[2 * TT][TT];        // their sums
    __shared__ float xs[NW][2 * TT][20];                    // X and Y by state row, then the c of both updates
    __shared__ float gate[2][TT];                           // alpha and beta
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, lg = lane >> 4;
    const int per = p.DV / DROWS, u = (int)blockIdx.x, sh = u / per;   // sequence * H + head
    const int s = sh / p.H, h = sh - s * p.H, r0 = (u - sh * per) * DROWS + 16 * wave;
    float* const rows = p.S + ((long)sh * p.DV + r0 + l16) * DK + 4 * lg;   // this lane's row
    int beg, end;
    seq_span(p.s, s, beg, end);
    const int kept = p.keep ? min(max(tab(p.keep, s), 0), end - beg) : end - beg, todo = p.q ? end - beg : kept;
    if (todo == 0) return;
    const int row = r0 + l16;
    const long hk = h / p.G;
    floatx4 S[NB];
    auto tile = [&](int t0, auto FIRST) {
        const int m = min(todo - t0, TT);
        const long tok = beg + t0;
        // Everything of the tokens is asked for ahead of the state, so that what they make among themselves is done by the time
        // it arrives (loads come back in order).
        constexpr int LPR = DK / 4, NK = 2 * TT * LPR / NT;   // 4 channels a thread, LPR neighbouring threads a row
        static_assert(2 * TT * LPR % NT == 0, "every thread has its share");
        floatx4 in[NK];
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            const int r = (tid + NT * i) / LPR, t = r % TT;
            in[i] = floatx4{0.f, 0.f, 0.f, 0.f};
            if (t < m && (r < TT || p.q)) in[i] = four((const IO*)(r < TT ? p.k : p.q) + ((tok + t) * p.HK + hk) * DK + 4 * (tid % LPR));
        }
        float gt = 0.f, v[TT];
        if (tid < 2 * TT && tid % TT < m) gt = (tid < TT ? p.g : p.beta)[(tok + tid % TT) * p.H + h];
#pragma unroll
        for (int t = 0; t < TT; ++t) v[t] = t < m ? to_f(((const IO*)p.v)[((tok + t) * p.H + h) * p.DV + row]) : 0.f;
        if constexpr (decltype(FIRST)::value) {
#pragma unroll
            for (int b = 0; b < NB; ++b) S[b] = f4(rows + 16 * b);
        } else {
            __syncthreads();   // (the tile before no longer reads the shared arrays)
        }
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            const int r = (tid + NT * i) / LPR;
            floatx4 x = in[i];
            if (p.pre & PRE_L2) {
                float ss = x[0] * x[0] + x[1] * x[1] + x[2] * x[2] + x[3] * x[3];
#pragma unroll
                for (int off = LPR / 2; off >= 1; off >>= 1) ss += __shfl_xor(ss, off, 64);
                x *= 1.f / sqrtf(ss + L2_EPS);
            }
            if (r >= TT) x *= p.scale;
            *reinterpret_cast<floatx4*>(&kq[r][4 * (tid % LPR)]) = x;
        }
        if (tid < TT) gate[0][tid] = tid < m ? expf((p.pre & PRE_GATES) ? gate_g(gt) : gt) : 1.f;
        else if (tid < 2 * TT) gate[1][tid - TT] = tid - TT < m ? ((p.pre & PRE_GATES) ? gate_beta(gt) : gt) : 0.f;
        lds_barrier();
        floatx4 own = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < NB; ++b)
            if (b % NW == wave) {   // (column i of the product with the keys and queries themselves: row i)
                const floatx4 a = f4(&kq[l16][16 * b + 4 * lg]);
#pragma unroll
                for (int e = 0; e < 4; ++e) own = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], a[e], own, 0, 0, 0);
            }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (l16 < TT) part[wave][4 * lg + e][l16] = own[e];
        lds_barrier();
        for (int i = tid; i < 2 * TT * TT; i += NT) {
            float y = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) y += part[w][i / TT][i % TT];
            pair[i / TT][i % TT] = y;
        }
        floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const floatx4 a = f4(&kq[l16][16 * b + 4 * lg]);
#pragma unroll
            for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], S[b][e], x, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) xs[wave][4 * lg + e][l16] = x[e];
        lds_barrier();
        // the tile's tokens, row by row
        float c[TT], ck[TT], gamma = 1.f, gamma_k = 1.f;
        const int kt = min(max(kept - t0, 0), TT);   // kept ones of the tile
#pragma unroll
        for (int t = 0; t < TT; ++t) c[t] = ck[t] = 0.f;
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            if (t >= m) break;
            const float al = gate[0][t];
            const floatx4 k0 = f4(&pair[t][0]), k1 = f4(&pair[t][4]);
            gamma *= al;
            float sk = gamma * xs[wave][t][l16];
#pragma unroll
            for (int i = 0; i < t; ++i) {
                c[i] *= al;
                sk += c[i] * (i < 4 ? k0[i] : k1[i - 4]);
            }
            c[t] = gate[1][t] * (v[t] - sk);
            if (p.q) {
                const floatx4 q0 = f4(&pair[TT + t][0]), q1 = f4(&pair[TT + t][4]);
                float o = gamma * xs[wave][TT + t][l16];
#pragma unroll
                for (int i = 0; i <= t; ++i) o += c[i] * (i < 4 ? q0[i] : q1[i - 4]);
                if (lane < 16) ((IO*)p.o)[((tok + t) * p.H + h) * p.DV + row] = from_f<IO>(o);
            }
            if (t + 1 == kt) {
                gamma_k = gamma;
#pragma unroll
                for (int i = 0; i <= t; ++i) ck[i] = c[i];
            }
        }
        const bool more = t0 + TT < todo, store = kt > 0 && t0 + kt == kept;
        if (!more && !store) return;
        // S' = gamma S + sum_i c_i k_i^T: first the kept state, then the next tile's
        __builtin_amdgcn_wave_barrier();
        if (lane < 16)
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                xs[wave][t][lane] = ck[t];
                xs[wave][TT + t][lane] = c[t];
            }
        __builtin_amdgcn_wave_barrier();
        auto update = [&](int first, float decay, int count, auto put) {
            float w[TT / 4];
#pragma unroll
            for (int z = 0; z < TT / 4; ++z) w[z] = xs[wave][first + 4 * z + lg][l16];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                float a[TT / 4];
#pragma unroll
                for (int z = 0; z < TT / 4; ++z) a[z] = 4 * z + lg < count ? kq[4 * z + lg][16 * b + l16] : 0.f;
                floatx4 y = S[b] * decay;
#pragma unroll
                for (int z = 0; z < TT / 4; ++z) y = __builtin_amdgcn_mfma_f32_16x16x4f32(a[z], w[z], y, 0, 0, 0);
                put(b, y);
            }
        };
        if (store) update(0, gamma_k, kt, [&](int b, floatx4 y) { *reinterpret_cast<floatx4*>(rows + 16 * b) = y; });
        if (more) update(TT, gamma, TT, [&](int b, floatx4 y) { S[b] = y; });
    };
    tile(0, Ic<1>{});
    for (int t0 = TT; t0 < todo; t0 += TT) tile(t0, Ic<0>{});
}

// ------------------------------------------------------------------ verification of drafts
// Token j of a sequence's drafts x_j is accepted while u_j q_j(x_j) < p_j(x_j), both sides exact in 64 bits (a product of two
// floats has 48).  Where the first is not, the next token is drawn from w = max(p_j - q_j, 0) of that row, behind the last
// draft from w = p of the row after it: the lowest v with w_0 + .. + w_v > u W, sums in 64 bits.  Their roundings are
// seen where u W falls as near to a border as they reach: a running sum passes 59 + 2 c additions on its way at most and W with
// its product by u 19 + c, c = V / 65536 rounded up (a lane's slices), so (78 + 3 c) 2^-53 of W, 2^-46 of it for a million tokens.
// w = p, too, where no w is positive.  Entries that are not positive and finite count as 0.
// k_verify_sums: a wave for each slice of VS tokens of the row that is left, their sum of w; k_verify_pick: the slice that holds
// u W, then the token in it.  Bound by the two rows' bytes: 64 sequences, rows of 131072 floats (67 MB, of which 54 came from
// memory and the rest from the last-level cache), 11.8 and 4.1 us; small calls by latency (drafts, their probabilities, the rows,
// the sums wait for one another): 3.5 and 2.9 for one of 50000.
// Waves that take several slices of a sequence, one after another, so that 24 (12) a CU are all there are, look the drafts up
// less often but wait longer: 96 rows of 100003 floats 16.8 (17.5) us a call against 16.4 of one each, 64 of 131072 in bf16 15.3 (17.7)
// against 13.2.  Slices of 512: 12.7 us for 96 rows of 100003 in bf16 (11.3 of 1024), 16.8 (16.3) of two in floats, but 5.8 (6.2) for
// one sequence; of 2048, 16.4 against 12.8 before the last step.
struct VerifyParams {
    const void* p;            // [n][m + 1][..], ps elements a row
    const void* q;            // [n][m][..], qs elements a row, or null: 1 for the drafted token
    const int32_t* drafts;    // [n][m]
    const int32_t* lens;      // or null: m
    const float* u;           // [n][m + 1]
    int32_t* tokens;          // [n][m + 1]
    int32_t* counts;          // [n]
    double* part;             // [n][slices] sums of w
    long ps, qs;
    int m, V, slices, groups;   // groups: workgroups of k_verify_sums a sequence
};
constexpr int VS = 1024;

__device__ __forceinline__ float probability(float x) { return __builtin_amdgcn_classf(x, 0x180) ? x : 0.f; }   // (positive, finite)

// The number of accepted drafts of sequence s, and of its drafts, by a whole wave.  (All m are looked up, also those past the sequence's number of
// drafts, so that it is loaded along with them and not ahead of them.)
template <typename IO> __device__ __forceinline__ int accepted(const VerifyParams& p, int s, int& len) {
    const int lane = threadIdx.x & 63;
    len = p.m;
    if (p.lens) len = p.lens[s];
    int first = p.m;
    for (int base = 0; base < p.m && first == p.m; base += 64) {
        const int j = base + lane;
        bool ok = true;
        if (j < p.m) {
            const int x = p.drafts[(long)s * p.m + j];
            ok = false;
            if (x >= 0 && x < p.V) {
                const double pr = probability(to_f(((const IO*)p.p)[((long)s * (p.m + 1) + j) * p.ps + x]));
                const double qr = p.q ? probability(to_f(((const IO*)p.q)[((long)s * p.m + j) * p.qs + x])) : 1.f;
                ok = (double)p.u[(long)s * (p.m + 1) + j] * qr < pr;
            }
        }
        const uint64_t no = __builtin_amdgcn_ballot_w64(!ok);
        if (no) first = base + __builtin_ctzll(no);
    }
    len = __builtin_amdgcn_readfirstlane(min(max(len, 0), p.m));
    return min(first, len);
}

// w of a row's entries: of row a of the target, less row a of the drafts'.
template <typename IO> struct Rest {
    const IO* p;
    const IO* q;   // null: nothing, but for
    int certain;   // the token whose draft was certain, or -1
};
template <typename IO> __device__ __forceinline__ Rest<IO> rest_of(const VerifyParams& p, int s, int a, int len) {
    Rest<IO> r;
    r.p = (const IO*)p.p + ((long)s * (p.m + 1) + a) * p.ps;
    r.q = a < len && p.q ? (const IO*)p.q + ((long)s * p.m + a) * p.qs : nullptr;
    r.certain = a < len && !p.q ? tab(p.drafts, (long)s * p.m + a) : -1;
    return r;
}

// w of tokens v0 + STEP i + e, i < N, e < 4 (0 from `end` on; whole: the wave has none there), all loads sent off before the first
// is used: without a branch between them, whose end would wait for what it has to convert (96 rows of 100003 in bf16 11.3 us a call,
// with a branch at every group of 4 12.8; less a second row 13.6 and 16.6).
template <typename IO, int N, int STEP> __device__ __forceinline__ void rest(const Rest<IO>& r, int v0, int end, bool whole, double (&w)[N][4]) {
    auto all = [&](auto WHOLE, auto LESS) {
        floatx4 x[N], y[N];
        auto load = [&](const IO* src, floatx4 (&z)[N]) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int v = v0 + STEP * i;
                if constexpr (decltype(WHOLE)::value) {
                    z[i] = four(src + v);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float one = to_f(src[min(v + e, end - 1)]);
                        z[i][e] = v + e < end ? one : 0.f;
                    }
                }
            }
        };
        load(r.p, x);
        if constexpr (decltype(LESS)::value) load(r.q, y);
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[i][e] = probability(x[i][e]);
                if constexpr (decltype(LESS)::value) w[i][e] = fmax(w[i][e] - (double)probability(y[i][e]), 0.);
            }
    };
    if (r.q) {
        if (whole) all(Ic<1>{}, Ic<1>{}); else all(Ic<0>{}, Ic<1>{});
        return;
    }
    if (whole) all(Ic<1>{}, Ic<0>{}); else all(Ic<0>{}, Ic<0>{});
    if (__builtin_amdgcn_ballot_w64(r.certain >= v0 && r.certain < v0 + STEP * (N - 1) + 4))
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (v0 + STEP * i + e == r.certain) w[i][e] = fmax(w[i][e] - 1., 0.);
}

constexpr int VE = VS / 64 / 4;   // groups of 4 tokens of a lane

// The sum of w over a slice, by a wave, in every lane.
template <typename IO> __device__ __forceinline__ double slice_sum(const Rest<IO>& r, int slice, int V) {
    const int lane = threadIdx.x & 63, first = slice * VS;
    double w[VE][4], sum = 0.;
    rest<IO, VE, 256>(r, first + 4 * lane, V, first + VS <= V, w);
#pragma unroll
    for (int i = 0; i < VE; ++i) sum += (w[i][0] + w[i][1]) + (w[i][2] + w[i][3]);
    return lane64(scan64(sum), 63);
}

template <typename IO>
__global__ __launch_bounds__(NT) void k_verify_sums(VerifyParams p) {
    const int s = (int)blockIdx.x / p.groups, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int w = ((int)blockIdx.x - s * p.groups) * (NT / 64) + wave;
    int len;
    const int a = accepted<IO>(p, s, len);
    const Rest<IO> r = rest_of<IO>(p, s, a, len);
    if (w < p.slices) {
        const double sum = slice_sum(r, w, p.V);
        if ((threadIdx.x & 63) == 0) p.part[(long)s * p.slices + w] = sum;
    }
    if (w == 0 && threadIdx.x == 0) p.counts[s] = a + 1;
}

template <typename IO>
__global__ __launch_bounds__(NT) void k_verify_pick(VerifyParams p) {
    const int s = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    double* part = p.part + (long)s * p.slices;
    const int per = (p.slices + 63) / 64;   // slices of a lane
    double sum, inc;
    auto load = [&] {
        sum = 0.;
        for (int i = lane * per; i < min((lane + 1) * per, p.slices); ++i) sum += part[i];
        inc = scan64(sum);
    };
    load();
    const int a = tab(p.counts, s) - 1, len = p.lens ? min(max(tab(p.lens, s), 0), p.m) : p.m;
    const float u = p.u[(long)s * (p.m + 1) + p.m];
    Rest<IO> r = rest_of<IO>(p, s, a, len);
    if (!(lane64(inc, 63) > 0.)) {   // no w is positive: p itself
        r.q = nullptr;
        r.certain = -1;
        __syncthreads();   // (every wave has read the sums)
        for (int i = wave; i < p.slices; i += NT / 64) {
            const double x = slice_sum(r, i, p.V);
            if (lane == 0) part[i] = x;
        }
        __syncthreads();
        load();
    }
    if (wave != 0) return;
    // 1 or more: past every running sum (which, added up in another order than W, may round past it ahead of the last token).  NaN: 0.
    const double goal = u >= 1.f ? (double)INFINITY : (u > 0.f ? (double)u : 0.) * lane64(inc, 63);
    // the first lane, slice and token whose running sum passes the goal; each time else the last that holds anything
    int token = -1;
    uint64_t any = __builtin_amdgcn_ballot_w64(sum > 0.), past = __builtin_amdgcn_ballot_w64(sum > 0. && inc > goal);
    if (any) {
        int l = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(any);
        double run = lane64(inc - sum, l), ahead = run;
        int slice = 0;
        for (int i = l * per; i < min((l + 1) * per, p.slices); ++i) {
            const double x = part[i];
            if (!(x > 0.)) continue;
            slice = i;
            ahead = run;
            run += x;
            if (run > goal) break;
        }
        slice = __builtin_amdgcn_readfirstlane(slice);
        const int first = slice * VS, v0 = first + 4 * VE * lane;
        double w[VE][4];
        rest<IO, VE, 4>(r, v0, p.V, first + VS <= p.V, w);
        sum = 0.;
#pragma unroll
        for (int i = 0; i < VE; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += w[i][e];
        double c = ahead + (scan64(sum) - sum);
        int hit = -1, mine = -1;
#pragma unroll
        for (int i = 0; i < VE; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                c += w[i][e];
                if (w[i][e] > 0.) {
                    mine = v0 + 4 * i + e;
                    if (hit < 0 && c > goal) hit = mine;
                }
            }
        any = __builtin_amdgcn_ballot_w64(mine >= 0);
        past = __builtin_amdgcn_ballot_w64(hit >= 0);
        token = past ? __builtin_amdgcn_readlane(hit, __builtin_ctzll(past)) : any ? __builtin_amdgcn_readlane(mine, 63 - __builtin_clzll(any)) : -1;
    }
    for (int j = lane; j <= p.m; j += 64) p.tokens[(long)s * (p.m + 1) + j] = j < a ? p.drafts[(long)s * p.m + j] : j == a ? token : -1;
}
