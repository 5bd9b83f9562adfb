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
// wait for one another.
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

// Position, and slot or -1, of a token that is the i-th of m new ones of sequence s.
__device__ __forceinline__ void map_token(const TablesParams& p, int t, int s, int i, int m) {
    const int pos = max(p.lens[s], 0) - m + i;
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

// The first index i of [0, n) with ends[i] > x (ends nondecreasing), n where there is none.
__device__ __forceinline__ int first_past(const int32_t* ends, int n, int x) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (ends[mid] > x) hi = mid; else lo = mid + 1;
    }
    return lo;
}

constexpr int NTA = 1024;   // threads of k_cache_tables, and sequences that it takes at a time
static_assert(NTA == NSU, "wg_scan's workgroup");

// maps: the positions and slots too (at most NTA sequences).
__global__ __launch_bounds__(NTA) void k_cache_tables(TablesParams p, int maps) {
    __shared__ int ends[NTA], at[NTA], cu_ends[NTA];   // running sums of pages moved, where they stand in a sequence's row; token offsets
    __shared__ int red[NTA / 64];
    const int tid = threadIdx.x, page = 1 << p.shift;
    auto sum = [](int a, int b) { return a + b; };
    const int rows = p.rows;
    auto tokens = [rows](int a, int b) { return min(a + b, rows); };   // (rows < 2^30)
    const int have = min(max(p.n_free[0], 0), p.n_pages);
    int held, target;   // of sequence base + tid
    auto load = [&](int i) {
        held = target = 0;
        if (i >= p.n) return;
        held = min(max(p.held[i], 0), p.max_pages);
        const int len = max(p.lens[i], 0);
        target = min((int)(((long)len + page - 1) >> p.shift), p.max_pages);
        if (p.shared) target = max(target, min(p.shared[i], held));
    };
    // pages given back (their sums stay below 2^31: n max_pages does)
    int given = 0, wanted = 0, token = 0, all;
    for (int base = 0; base < p.n; base += NTA) {
        const int i = base + tid, m = min(p.n - base, NTA);
        load(i);
        const int give = max(held - target, 0), y = wg_scan(give, sum, red, all);
        ends[tid] = y;
        at[tid] = target - (y - give);
        const int total = all;
        wg_scan(max(target - held, 0), sum, red, all);
        wanted += all;
        if (p.new_lens) {
            const int e = tokens(token, wg_scan(i < p.n ? min(max(p.new_lens[i], 0), rows) : 0, tokens, red, all));
            if (i < p.n) {
                cu_ends[tid] = e;
                p.cu[i + 1] = e;
            }
            token = tokens(token, all);
        } else if (i < p.n && p.cu) {
            p.cu[i + 1] = (i + 1) * (rows / p.n);
        }
        __syncthreads();
        for (int x = tid; x < total; x += NTA) {
            const int s = first_past(ends, m, x);
            int32_t* entry = p.table + (long)(base + s) * p.max_pages + at[s] + x;
            const int to = have + given + x;
            if (to < p.n_pages) p.free[to] = *entry;
            *entry = -1;
        }
        given += total;
        __syncthreads();
    }
    if (tid == 0 && p.cu) p.cu[0] = 0;
    const int pool = min(have + given, p.n_pages), got = min(wanted, pool);
    // pages taken
    int taken = 0;
    for (int base = 0; base < p.n; base += NTA) {
        const int i = base + tid, m = min(p.n - base, NTA);
        if (p.n > NTA) load(i);
        const int take = max(target - held, 0), y = wg_scan(take, sum, red, all);
        ends[tid] = y;
        at[tid] = held - (y - take);
        if (i < p.n) p.held[i] = min(held, target) + min(max(got - taken - (y - take), 0), take);
        const int total = all;
        __syncthreads();
        for (int x = tid; x < total; x += NTA) {
            const int s = first_past(ends, m, x);
            p.table[(long)(base + s) * p.max_pages + at[s] + x] = taken + x < got ? p.free[pool - got + taken + x] : -1;
        }
        taken += total;
        __syncthreads();
    }
    if (tid == 0) {
        p.n_free[0] = pool - got;
        if (p.missing) p.missing[0] = wanted - got;
    }
    if (!maps) return;
    const int T = rows / p.n;
    for (int t = tid; t < rows; t += NTA) {
        if (!p.new_lens) {
            map_token(p, t, t / T, t % T, T);
            continue;
        }
        const int s = first_past(cu_ends, p.n, t);
        if (s >= p.n) {
            map_none(p, t);
        } else {
            const int beg = s > 0 ? cu_ends[s - 1] : 0;
            map_token(p, t, s, t - beg, cu_ends[s] - beg);
        }
    }
}

// The positions and slots of many tokens, from the tables and offsets that k_cache_tables left.
__global__ __launch_bounds__(NT) void k_cache_maps(TablesParams p) {
    const int t = (int)blockIdx.x * NT + threadIdx.x;
    if (t >= p.rows) return;
    if (!p.new_lens) {
        const int T = p.rows / p.n;
        map_token(p, t, t / T, t % T, T);
        return;
    }
    const int s = first_past(p.cu + 1, p.n, t);
    if (s >= p.n) {
        map_none(p, t);
        return;
    }
    const int beg = p.cu[s];
    map_token(p, t, s, t - beg, p.cu[s + 1] - beg);
}

// ------------------------------------------------------------------ k_draft_step
// A few tokens of each sequence through a recurrent layer (the recurrence at the head of gdn.hip), the state read once and
// written, where any token is kept, once.  In tiles of TT = 8 tokens, with S the state before the tile:
//   X_t = S k_t,  Y_t = S (scale q_t)                       one product [K; Q] S^T of 16 rows, fp32 matrix instructions
//   u_t = beta_t (v_t - gamma_t X_t - sum_{i<t} c_i (k_t . k_i)),   c_i = u_i decayed from i to t
//   o_t = gamma_t Y_t + sum_{i<=t} c_i (q_t . k_i)          row by row of the state, one lane a row
//   S'  = gamma_n S + sum_i c_i k_i^T                       c after the n-th token: the next tile's state, or the kept one
// Decays multiply as the tokens pass, so that a gate of 0 (log-decay -inf) is one; nothing is divided.
// A wave holds 16 RT state rows in registers as accumulators of S^T tiles: lane 16 lg + j has row j's channels 16 b + 4 lg .. + 3,
// which is the layout of a product's operand and result alike, so S enters and leaves them without a move.
// Bound by memory (the state once in, and once out where tokens are kept).
constexpr int TT = 8;
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

template <typename IO, int DK, int RT, int NW>
__global__ __launch_bounds__(64 * NW) void k_draft_step(DraftParams p) {
    constexpr int NB = DK / 16, ROWS = 16 * RT * NW, N = 64 * NW, PITCH = DK + 4;
    __shared__ __align__(16) float kq[2 * TT][PITCH];       // keys, then queries, of the tile
    __shared__ __align__(16) float pair[NW][2 * TT][TT];    // a wave's share of k_t . k_i and q_t . k_i
    __shared__ __align__(16) float xs[NW][2 * TT][16 * RT]; // X and Y by state row, then the c of both updates
    __shared__ float gate[2][TT];                           // alpha and beta
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, lg = lane >> 4;
    const int per = p.DV / ROWS, u = (int)blockIdx.x, sh = u / per;   // sequence * H + head
    const int s = sh / p.H, h = sh - s * p.H, r0 = (u - sh * per) * ROWS + 16 * RT * wave;
    int beg, end;
    seq_span(p.s, s, beg, end);
    const int kept = p.keep ? min(max(tab(p.keep, s), 0), end - beg) : end - beg, todo = p.q ? end - beg : kept;
    if (todo == 0) return;
    float* const rows = p.S + ((long)sh * p.DV + r0 + l16) * DK + 4 * lg;   // of tile 0: this lane's row
    floatx4 S[RT][NB];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int b = 0; b < NB; ++b) S[t][b] = f4(rows + (long)16 * t * DK + 16 * b);
    const int row = r0 + lane % (16 * RT);   // the row that this lane works out
    const long hk = h / p.G;
    for (int t0 = 0; t0 < todo; t0 += TT) {
        const int m = min(todo - t0, TT);
        const long tok = beg + t0;
        float v[TT];
#pragma unroll
        for (int t = 0; t < TT; ++t) v[t] = t < m ? to_f(((const IO*)p.v)[((tok + t) * p.H + h) * p.DV + row]) : 0.f;
        __syncthreads();   // (the tile before no longer reads these)
        // keys and queries, 4 channels a thread, DK / 4 neighbouring threads a row
        constexpr int LPR = DK / 4;
#pragma unroll
        for (int i = tid; i < 2 * TT * LPR; i += N) {
            const int r = i / LPR, c = 4 * (i % LPR), t = r % TT;
            floatx4 x = {0.f, 0.f, 0.f, 0.f};
            if (t < m && (r < TT || p.q)) {
                const IO* src = (const IO*)(r < TT ? p.k : p.q) + ((tok + t) * p.HK + hk) * DK + c;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = to_f(src[e]);
            }
            if (p.pre & PRE_L2) {
                float ss = x[0] * x[0] + x[1] * x[1] + x[2] * x[2] + x[3] * x[3];
#pragma unroll
                for (int off = LPR / 2; off >= 1; off >>= 1) ss += __shfl_xor(ss, off, 64);
                x *= 1.f / sqrtf(ss + L2_EPS);
            }
            if (r >= TT) x *= p.scale;
            *reinterpret_cast<floatx4*>(&kq[r][c]) = x;
        }
        if (tid < 2 * TT) {
            const int t = tid % TT;
            const long at = (tok + t) * p.H + h;
            if (tid < TT)
                gate[0][t] = t < m ? expf((p.pre & PRE_GATES) ? gate_g(p.g[at]) : p.g[at]) : 1.f;
            else
                gate[1][t] = t < m ? ((p.pre & PRE_GATES) ? gate_beta(p.beta[at]) : p.beta[at]) : 0.f;
        }
        __syncthreads();
        floatx4 x[RT], own = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < RT; ++t) x[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const floatx4 a = f4(&kq[l16][16 * b + 4 * lg]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int t = 0; t < RT; ++t) x[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], S[t][b][e], x[t], 0, 0, 0);
            if (b % NW == wave)   // (column i of the product with the keys and queries themselves: row i)
#pragma unroll
                for (int e = 0; e < 4; ++e) own = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], a[e], own, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (l16 < TT) pair[wave][4 * lg + e][l16] = own[e];
#pragma unroll
            for (int t = 0; t < RT; ++t) xs[wave][4 * lg + e][16 * t + l16] = x[t][e];
        }
        __syncthreads();
        // the tile's tokens, row by row
        float c[TT], ck[TT], gamma = 1.f, gamma_k = 1.f;
        const int kt = min(max(kept - t0, 0), TT);   // kept ones of the tile
        const int lr = lane % (16 * RT);
#pragma unroll
        for (int t = 0; t < TT; ++t) ck[t] = 0.f;
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const float al = gate[0][t];
            float kk[TT], qk[TT];
#pragma unroll
            for (int i = 0; i <= t; ++i) {
                kk[i] = qk[i] = 0.f;
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    kk[i] += pair[w][t][i];
                    qk[i] += pair[w][TT + t][i];
                }
            }
            gamma *= al;
            float sk = gamma * xs[wave][t][lr];
#pragma unroll
            for (int i = 0; i < t; ++i) {
                c[i] *= al;
                sk += c[i] * kk[i];
            }
            c[t] = gate[1][t] * (v[t] - sk);
            if (t < m && p.q) {
                float o = gamma * xs[wave][TT + t][lr];
#pragma unroll
                for (int i = 0; i <= t; ++i) o += c[i] * qk[i];
                if (lane < 16 * RT) ((IO*)p.o)[((tok + t) * p.H + h) * p.DV + row] = from_f<IO>(o);
            }
            if (t + 1 == kt) {
                gamma_k = gamma;
#pragma unroll
                for (int i = 0; i <= t; ++i) ck[i] = c[i];
            }
        }
        const bool more = t0 + TT < todo, store = kt > 0 && t0 + kt == kept;
        if (!more && !store) continue;
        // S' = gamma S + sum_i c_i k_i^T: first the kept state, then the next tile's
        __builtin_amdgcn_wave_barrier();
        if (lane < 16 * RT)
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                xs[wave][t][lane] = ck[t];
                xs[wave][TT + t][lane] = c[t];
            }
        __builtin_amdgcn_wave_barrier();
        auto update = [&](int first, float decay, int count, auto put) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                float a[TT / 4];
#pragma unroll
                for (int z = 0; z < TT / 4; ++z) a[z] = 4 * z + lg < count ? kq[4 * z + lg][16 * b + l16] : 0.f;
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    floatx4 y = S[t][b] * decay;
#pragma unroll
                    for (int z = 0; z < TT / 4; ++z)
                        y = __builtin_amdgcn_mfma_f32_16x16x4f32(a[z], xs[wave][first + 4 * z + lg][16 * t + l16], y, 0, 0, 0);
                    put(t, b, y);
                }
            }
        };
        if (store) update(0, gamma_k, kt, [&](int t, int b, floatx4 y) { *reinterpret_cast<floatx4*>(rows + (long)16 * t * DK + 16 * b) = y; });
        if (more) update(TT, gamma, TT, [&](int t, int b, floatx4 y) { S[t][b] = y; });
    }
}

// ------------------------------------------------------------------ verification of drafts
// Token j of a sequence's drafts x_j is accepted while u_j q_j(x_j) < p_j(x_j), both sides exact in 64 bits (a product of two
// floats has 48).  Where the first is not, the next token is drawn from w = max(p_j - q_j, 0) of that row, behind the last
// draft from w = p of the row after it: the lowest v with w_0 + .. + w_v > u W, sums in 64 bits, so that no rounding of
// theirs is seen but where u W falls within 2^-50 of a border.  w = p, too, where no w is positive.  Entries that are not
// positive and finite count as 0.
// k_verify_sums: a workgroup per slice of VS tokens of the row that is left, its sums of w and of p; k_verify_pick: the slice
// that holds u W, then the token in it.  Bound by the two rows' bytes.
struct VerifyParams {
    const void* p;            // [n][m + 1][..], ps elements a row
    const void* q;            // [n][m][..], qs elements a row, or null: 1 for the drafted token
    const int32_t* drafts;    // [n][m]
    const int32_t* lens;      // or null: m
    const float* u;           // [n][m + 1]
    int32_t* tokens;          // [n][m + 1]
    int32_t* counts;          // [n]
    double2* part;            // [n][slices] sums of w and of p
    long ps, qs;
    int m, V, slices;
};
constexpr int VS = 4096;

__device__ __forceinline__ float probability(float x) { return x > 0.f && x <= -LOWEST ? x : 0.f; }

// The number of accepted drafts of sequence s, and of its drafts, by a whole wave.
template <typename IO> __device__ __forceinline__ int accepted(const VerifyParams& p, int s, int& len) {
    const int lane = threadIdx.x & 63;
    len = p.lens ? min(max(tab(p.lens, s), 0), p.m) : p.m;
    for (int base = 0; base < len; base += 64) {
        const int j = base + lane;
        bool ok = true;
        if (j < len) {
            const int x = p.drafts[(long)s * p.m + j];
            ok = false;
            if (x >= 0 && x < p.V) {
                const double pr = probability(to_f(((const IO*)p.p)[((long)s * (p.m + 1) + j) * p.ps + x]));
                const double qr = p.q ? probability(to_f(((const IO*)p.q)[((long)s * p.m + j) * p.qs + x])) : 1.f;
                ok = (double)p.u[(long)s * (p.m + 1) + j] * qr < pr;
            }
        }
        const uint64_t no = __builtin_amdgcn_ballot_w64(!ok);
        if (no) return base + __builtin_ctzll(no);
    }
    return len;
}

// w of a row's entries: of row a of the target, less row a of the drafts' where `less`.
template <typename IO> struct Rest {
    const IO* p;
    const IO* q;
    int certain;   // the token whose draft was certain (q null), or -1
    __device__ __forceinline__ double w(int v, double pr) const {
        const double qr = q ? probability(to_f(q[v])) : v == certain ? 1. : 0.;
        return pr > qr ? pr - qr : 0.;
    }
    __device__ __forceinline__ double target(int v) const { return probability(to_f(p[v])); }
};
template <typename IO> __device__ __forceinline__ Rest<IO> rest_of(const VerifyParams& p, int s, int a, int len) {
    Rest<IO> r;
    r.p = (const IO*)p.p + ((long)s * (p.m + 1) + a) * p.ps;
    r.q = a < len && p.q ? (const IO*)p.q + ((long)s * p.m + a) * p.qs : nullptr;
    r.certain = a < len && !p.q ? tab(p.drafts, (long)s * p.m + a) : -1;
    return r;
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) x += __shfl_xor(x, off, 64);
    return x;
}

template <typename IO>
__global__ __launch_bounds__(NT) void k_verify_sums(VerifyParams p) {
    __shared__ double2 red[NT / 64];
    const int s = (int)blockIdx.x / p.slices, slice = (int)blockIdx.x - s * p.slices, tid = threadIdx.x;
    int len;
    const int a = accepted<IO>(p, s, len);
    const Rest<IO> r = rest_of<IO>(p, s, a, len);
    double sw = 0., sp = 0.;
    const int first = slice * VS, end = min(first + VS, p.V);
    for (int v = first + tid; v < end; v += NT) {
        const double pr = r.target(v);
        sp += pr;
        sw += r.w(v, pr);
    }
    sw = wave_sum(sw);
    sp = wave_sum(sp);
    if ((tid & 63) == 0) red[tid >> 6] = double2{sw, sp};
    __syncthreads();
    if (tid != 0) return;
    double2 y = red[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) {
        y.x += red[w].x;
        y.y += red[w].y;
    }
    p.part[blockIdx.x] = y;
}

template <typename IO>
__global__ __launch_bounds__(NT) void k_verify_pick(VerifyParams p) {
    __shared__ double before[NT / 64];
    __shared__ int found, last;
    const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int len;
    const int a = accepted<IO>(p, s, len);
    const Rest<IO> r = rest_of<IO>(p, s, a, len);
    const double2* part = p.part + (long)s * p.slices;
    double W = 0., P = 0.;   // (every thread the same sums, in order)
    for (int i = 0; i < p.slices; ++i) {
        W += part[i].x;
        P += part[i].y;
    }
    const bool plain = !(W > 0.);
    const double all = plain ? P : W;
    const float draw = p.u[(long)s * (p.m + 1) + p.m];
    const double goal = (draw > 0.f ? (double)draw : 0.) * all;   // (NaN: 0)
    // the first slice whose running sum passes the goal; else the last one that holds anything
    int slice = -1;
    double run = 0., ahead = 0.;
    for (int i = 0; i < p.slices; ++i) {
        const double x = plain ? part[i].y : part[i].x;
        if (!(x > 0.)) continue;
        slice = i;
        ahead = run;
        run += x;
        if (run > goal) break;
    }
    if (tid == 0) {
        found = 1 << 30;
        last = -1;
    }
    __syncthreads();
    int token = -1;
    if (slice >= 0) {
        constexpr int EACH = VS / NT;
        const int v0 = slice * VS + tid * EACH;
        double w[EACH], sum = 0.;
        int mine = -1;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            w[e] = 0.;
            if (v0 + e < p.V) {
                const double pr = r.target(v0 + e);
                w[e] = plain ? pr : r.w(v0 + e, pr);
            }
            sum += w[e];
            if (w[e] > 0.) mine = v0 + e;
        }
        double inc = sum;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const double y = __shfl_up(inc, off, 64);
            if (lane >= off) inc += y;
        }
        if (lane == 63) before[wave] = inc;
        __syncthreads();
        double c = ahead;
        for (int z = 0; z < wave; ++z) c += before[z];
        c += inc - sum;
        int hit = -1;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            c += w[e];
            if (hit < 0 && w[e] > 0. && c > goal) hit = v0 + e;
        }
        if (hit >= 0) atomicMin(&found, hit);
        if (mine >= 0) atomicMax(&last, mine);
        __syncthreads();
        token = found < 1 << 30 ? found : last;
    }
    for (int j = tid; j <= p.m; j += NT) p.tokens[(long)s * (p.m + 1) + j] = j < a ? p.drafts[(long)s * p.m + j] : j == a ? token : -1;
    if (tid == 0) p.counts[s] = a + 1;
}
