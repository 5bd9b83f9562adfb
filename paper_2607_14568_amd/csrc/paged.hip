// The attention layers' serving operators (included by gdn.hip): the norm and rotation of a prompt's queries and keys,
// the new tokens' keys and values into a paged cache, and the new tokens' attention over it.
//
// A step brings n new tokens to each sequence; seq_lens[s] counts the tokens of sequence s with them, so that its i-th
// new token stands at position seq_lens[s] - n + i.  Position p lives in page block_table[s][p / page], slot p % page, of
// a cache [n_pages][H_kv][page][d]: the rows of a page and head lie together, page * d elements that one workgroup streams.

// ------------------------------------------------------------------ sequences of a step
struct StepSeqs {
    const int32_t* cu;    // packed: offsets [n + 1] of the new tokens; null: T tokens each
    const int32_t* lens;  // tokens with the new ones [n]; null: no cache (positions from 0)
    int n, T;             // sequences; tokens of a dense sequence (packed: of the call)
};

// The tokens [beg, end) of the call that are new in sequence base + lane (none past the last sequence).  Called by a whole
// wave, with base = 0, 64, .. and `at` (0 at first) carried along.  Packed offsets outside the contract are clamped into
// a nondecreasing partition of [0, T].
__device__ __forceinline__ void span64(const StepSeqs& q, int base, int& at, int& beg, int& end) {
    const int lane = threadIdx.x & 63, j = base + lane;
    if (!q.cu) {
        beg = min(j, q.n) * q.T;
        end = min(j + 1, q.n) * q.T;
        return;
    }
    end = j < q.n ? min(max(q.cu[j + 1], at), q.T) : at;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(end, off, 64);
        if (lane >= off) end = max(end, y);
    }
    const int y = __shfl_up(end, 1, 64);
    beg = lane > 0 ? y : at;
    at = __builtin_amdgcn_readlane(end, 63);
}

// Sequence of token t of the call (a scalar), its place i among the sequence's new tokens and their number n; false for
// tokens behind the last sequence.  Called by a whole wave.
__device__ __forceinline__ bool step_seq(const StepSeqs& q, int t, int& s, int& i, int& n) {
    if (!q.cu) {
        s = t / q.T;
        i = t % q.T;
        n = q.T;
        return true;
    }
    int at = 0, beg, end;
    for (int base = 0; base < q.n; base += 64) {
        span64(q, base, at, beg, end);
        const uint64_t past = __builtin_amdgcn_ballot_w64(end > t);
        if (past) {
            const int l = __builtin_ctzll(past);
            const int b = __builtin_amdgcn_readlane(beg, l);
            s = base + l;
            i = t - b;
            n = __builtin_amdgcn_readlane(end, l) - b;
            return true;
        }
    }
    return false;
}

// ------------------------------------------------------------------ norm and rotation of a row
// A row of DH channels lies over DH / 8 neighbouring lanes, chunk c = lane % (DH / 8) holding channels 8 c .. 8 c + 7.
struct Turn {
    const double* freq;   // angle per position of pair i (rot / 2 of them), or null: no rotation
    int rot;              // channels that rotate, a multiple of 16
    int near;             // pairs (2 i, 2 i + 1); else (i, i + rot / 2)
    float eps;
};

// cos and sin of pos * freq[i], the angle in float64 (a float32 product is off by 2^-24 of an angle of up to 10^5
// radians), reduced there to within half a turn before it is rounded
__device__ __forceinline__ void angle(const Turn& t, int i, double pos, float& cs, float& sn) {
    double a = pos * t.freq[i] * 0.15915494309189535;
    a -= rint(a);
    sincospif((float)(2 * a), &sn, &cs);
}

// the angles of a chunk's 8 channels
__device__ __forceinline__ void angles(const Turn& t, int c, int pos, float (&cs)[8], float (&sn)[8]) {
    if (8 * c >= t.rot) {
#pragma unroll
        for (int e = 0; e < 8; ++e) { cs[e] = 1.f; sn[e] = 0.f; }
        return;
    }
    if (t.near) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            angle(t, 4 * c + e / 2, pos, cs[e], sn[e]);
            cs[e + 1] = cs[e];
            sn[e + 1] = sn[e];
            sn[e] = -sn[e];
        }
        return;
    }
    const int hc = t.rot / 16, first = c < hc;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        angle(t, 8 * (first ? c : c - hc) + e, pos, cs[e], sn[e]);
        if (first) sn[e] = -sn[e];
    }
}

// x: this lane's 8 channels; w: their weights or null; cs, sn: from angles() (used when t.freq).  y = x w / sqrt(mean(x^2)
// + eps), then (a, b) -> (a cos - b sin, b cos + a sin) over the pairs: every channel is x cs + partner sn.
template <int DH>
__device__ __forceinline__ void turn_row(const Turn& t, const float* w, const float (&cs)[8], const float (&sn)[8], float (&x)[8]) {
    constexpr int LPR = DH / 8;
    const int lane = threadIdx.x & 63, c = lane % LPR;
    if (w) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += x[e] * x[e];
#pragma unroll
        for (int off = 1; off < LPR; off <<= 1) ss += __shfl_xor(ss, off, 64);
        const float r = 1.f / sqrtf(ss * (1.f / DH) + t.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= r * w[8 * c + e];
    }
    if (t.freq) {
        const int hc = t.rot / 16;
        const int from = t.near ? lane : c < hc ? lane + hc : c < 2 * hc ? lane - hc : lane;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = t.near ? x[e ^ 1] : __shfl(x[e], from, 64);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * cs[e] + y[e] * sn[e];
    }
}

template <typename IO> __device__ __forceinline__ void load8(const IO* p, float (&x)[8]) {
    if constexpr (sizeof(IO) == 2) {
        const short8 v = *reinterpret_cast<const short8*>(p);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = bf(v[e]);
    } else {
        const floatx4 a = f4(p), b = f4(p + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[4 + e] = b[e]; }
    }
}
template <typename IO> __device__ __forceinline__ void store8(IO* p, const float (&x)[8]) {
    const floatx4 a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
    if constexpr (sizeof(IO) == 2) {
        *reinterpret_cast<bf16x8*>(p) = pack_bf16(a, b);
    } else {
        *reinterpret_cast<floatx4*>(p) = a;
        *reinterpret_cast<floatx4*>(p + 4) = b;
    }
}

// ------------------------------------------------------------------ the cache
struct Cache {
    void* k;              // [n_pages][HKV][page][d], bf16 or e4m3
    void* v;
    float* ks;            // e4m3: scales [n_pages][HKV]
    float* vs;
    const int32_t* table; // [n_seqs][max_pages]
    int n_pages, max_pages, page, shift;   // page = 1 << shift
};

// Page of block b of sequence s, or -1 when the table holds none there (b past it, or an entry outside the cache).
__device__ __forceinline__ int page_of(const Cache& c, int s, long b) {
    if (b < 0 || b >= c.max_pages) return -1;
    const int id = c.table[(long)s * c.max_pages + b];
    return id >= 0 && id < c.n_pages ? id : -1;
}

// ------------------------------------------------------------------ k_rows: tokens' rows, normed and rotated
// One wave takes `per` groups of 64 / (DH / 8) rows of one token: its q heads, its k heads and, into a bf16 cache, its v
// heads (those as they are).  Bound by memory: every row is read once and written once.
struct RowsParams {
    const void* q;
    const void* k;
    const void* v;
    void* qo;             // [tokens][H][d]
    void* ko;             // [tokens][HKV][d]; null: k goes to the cache
    long qs, ks, vs;      // elements from one token's row to the next
    int H, HKV;
    long tokens;
    int units, per;       // waves per token, row groups per wave
    const float* qw;
    const float* kw;
    const int32_t* pos;   // positions of the tokens; null: by the sequences
    Turn t;
    StepSeqs s;
    Cache c;
};

template <typename IO, int DH>
__device__ __forceinline__ void token_rows(const RowsParams& p, long wave) {
    constexpr int LPR = DH / 8, RPG = 64 / LPR;
    const long tok = wave / p.units;
    const int unit = (int)(wave % p.units), lane = threadIdx.x & 63, c = lane % LPR;
    if (tok >= p.tokens) return;
    int s = 0, i = 0, n = 0;
    if (!step_seq(p.s, tok, s, i, n)) return;
    const int pos = p.pos ? p.pos[tok] : p.s.lens ? p.s.lens[s] - n + i : i;
    float cs[8], sn[8];
    if (p.t.freq) angles(p.t, c, pos, cs, sn);
    const int HQ = p.q ? p.H : 0, rows = HQ + (p.k ? p.HKV : 0) + (p.v ? p.HKV : 0);
    const int id = p.k && !p.ko && pos >= 0 ? page_of(p.c, s, pos >> p.c.shift) : -1;
    for (int g = 0; g < p.per; ++g) {
        const int j = (unit * p.per + g) * RPG + lane / LPR;
        const int kind = j < HQ ? 0 : j < HQ + p.HKV ? 1 : 2;   // q, k, v
        const int h = kind == 0 ? j : kind == 1 ? j - HQ : j - HQ - p.HKV;
        const IO* src = kind == 0 ? (const IO*)p.q + tok * p.qs : kind == 1 ? (const IO*)p.k + tok * p.ks : (const IO*)p.v + tok * p.vs;
        float x[8] = {};
        if (j < rows) load8(src + h * DH + 8 * c, x);
        if (kind < 2) {
            // (a row's lanes share their kind, and the exchanges stay inside a row)
            turn_row<DH>(p.t, kind == 0 ? p.qw : p.kw, cs, sn, x);
        }
        if (j >= rows) continue;
        if (kind == 0) {
            store8((IO*)p.qo + (tok * p.H + h) * DH + 8 * c, x);
        } else if (p.ko) {
            store8((IO*)p.ko + (tok * p.HKV + h) * DH + 8 * c, x);
        } else if (id >= 0) {
            IO* base = (IO*)(kind == 1 ? p.c.k : p.c.v);
            store8(base + (((long)id * p.HKV + h) * p.c.page + (pos & (p.c.page - 1))) * DH + 8 * c, x);
        }
    }
}

template <typename IO, int DH>
__global__ __launch_bounds__(NT) void k_rows(RowsParams p) {
    token_rows<IO, DH>(p, (long)blockIdx.x * (NT / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
}

// ------------------------------------------------------------------ k_append_e4m3
// e4m3 codes with one scale per page and head, the smallest power of two s >= 2^-100 with every finite value at most 448 s
// (448: the type's largest).  A power of two costs a floating type no precision, and a page that later needs a larger
// scale has its codes brought to it exactly, but for those that become subnormal (under 2^-15 of the page's largest).
__device__ __forceinline__ float power_scale(float amax) {
    const uint32_t u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u);   // biased; 448 = 1.75 2^8
    return __uint_as_float((uint32_t)max(e, 27) << 23);
}
__device__ __forceinline__ uint64_t to_e4m3(const float (&x)[8], float inv) {   // round to nearest even; not finite: NaN
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = fabsf(x[e]) <= 3.402823466e38f ? x[e] * inv : __uint_as_float(0x7fc00000u);
    int a = 0, b = 0;
    a = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], a, false);
    a = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], a, true);
    b = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], b, false);
    b = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], b, true);
    return (uint64_t)(uint32_t)a | (uint64_t)(uint32_t)b << 32;
}
__device__ __forceinline__ void from_e4m3(uint64_t codes, float (&x)[8]) {
    typedef float floatx2 __attribute__((ext_vector_type(2)));
    const int a = (int)(uint32_t)codes, b = (int)(uint32_t)(codes >> 32);
    const floatx2 y[4] = {__builtin_amdgcn_cvt_pk_f32_fp8(a, false), __builtin_amdgcn_cvt_pk_f32_fp8(a, true),
                          __builtin_amdgcn_cvt_pk_f32_fp8(b, false), __builtin_amdgcn_cvt_pk_f32_fp8(b, true)};
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = y[e / 2][e % 2];
}

// The block-th page that the step's new tokens touch, over all sequences: its sequence s, the page's index b in it, the
// positions [first, len) of the sequence's new tokens and the call's row of the first of them.  Called by a whole wave;
// false past the last.
__device__ __forceinline__ bool touched_block(const StepSeqs& q, int shift, long block, int& s, int& b, int& first, int& len, int& row) {
    const int lane = threadIdx.x & 63;
    int at = 0, beg, end;
    long before = 0;
    for (int base = 0; base < q.n; base += 64) {
        span64(q, base, at, beg, end);
        const int L = base + lane < q.n ? q.lens[base + lane] : 0;
        const int f = max(L - (end - beg), 0);   // (a token before position 0 is not written)
        const int cnt = end > beg && L > 0 ? ((L - 1) >> shift) - (f >> shift) + 1 : 0;
        long sum = cnt;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const long y = __shfl_up(sum, off, 64);
            if (lane >= off) sum += y;
        }
        const uint64_t past = __builtin_amdgcn_ballot_w64(before + sum > block);
        if (past) {
            const int l = __builtin_ctzll(past);
            s = base + l;
            first = __builtin_amdgcn_readlane(f, l);
            len = __builtin_amdgcn_readlane(L, l);
            b = (first >> shift) + (int)(block - before) + __builtin_amdgcn_readlane(cnt, l) - (int)__shfl(sum, l, 64);
            b = __builtin_amdgcn_readfirstlane(b);
            row = __builtin_amdgcn_readlane(end, l) - (len - first);
            return true;
        }
        before += __shfl(sum, 63, 64);
    }
    return false;
}

// One workgroup per (touched page, head, K or V), after `row_wgs` workgroups of the q rows.  It holds the page's new
// tokens in registers, finds their largest value, and writes codes and scale.
template <int DH, int IT>   // IT: passes of NT / (DH / 8) rows over a page
__global__ __launch_bounds__(NT) void k_append_e4m3(RowsParams p, int row_wgs) {
    constexpr int LPR = DH / 8, RPP = NT / LPR;
    __shared__ float red[NT / 64];
    const int tid = threadIdx.x, c = tid % LPR, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if ((int)blockIdx.x < row_wgs) {
        RowsParams r = p;
        r.k = r.v = nullptr;
        token_rows<bf16_t, DH>(r, (long)blockIdx.x * (NT / 64) + wave);
        return;
    }
    const long u = (long)blockIdx.x - row_wgs;
    const int is_v = (int)(u & 1), h = (int)(u / 2 % p.HKV);
    int s, b, first, len, row;
    if (!touched_block(p.s, p.c.shift, u / 2 / p.HKV, s, b, first, len, row)) return;
    const int id = page_of(p.c, s, b);
    if (id < 0) return;
    const long at0 = (long)b << p.c.shift;   // position of the page's first slot
    const int lo = (int)max(first - at0, 0L), hi = (int)min(len - at0, (long)p.c.page);   // its new slots
    const bf16_t* src = (const bf16_t*)(is_v ? p.v : p.k) + h * DH + 8 * c;
    const long stride = is_v ? p.vs : p.ks;
    float x[IT][8], amax = 0.f;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        const int r = it * RPP + tid / LPR;
        const bool in = r >= lo && r < hi;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[it][e] = 0.f;
        if (in) load8(src + (row + (at0 + r - first)) * stride, x[it]);
    }
    if (!is_v) {
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            if (it * RPP >= hi || (it + 1) * RPP <= lo) continue;   // (the whole workgroup's)
            float cs[8], sn[8];
            if (p.t.freq) angles(p.t, c, (int)at0 + it * RPP + tid / LPR, cs, sn);
            turn_row<DH>(p.t, p.kw, cs, sn, x[it]);
        }
    }
#pragma unroll
    for (int it = 0; it < IT; ++it)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float m = fabsf(x[it][e]);
            amax = fmaxf(amax, m <= 3.402823466e38f ? m : 0.f);
        }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) amax = fmaxf(amax, __shfl_xor(amax, off, 64));
    if ((tid & 63) == 0) red[wave] = amax;
    __syncthreads();
    amax = red[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) amax = fmaxf(amax, red[w]);
    float scale = power_scale(amax);
    float* ps = (is_v ? p.c.vs : p.c.ks) + (long)id * p.HKV + h;
    uint8_t* codes = (uint8_t*)(is_v ? p.c.v : p.c.k) + ((long)id * p.HKV + h) * p.c.page * DH + 8 * c;
    if (lo > 0) {   // the page holds earlier tokens of the sequence, in its old scale
        const float old = *ps;
        if (old >= scale) {
            scale = old;
        } else {
            const float ratio = old / scale;
            for (int r = tid / LPR; r < lo; r += RPP) {
                uint64_t* at = (uint64_t*)(codes + r * DH);
                float y[8];
                from_e4m3(*at, y);
                *at = to_e4m3(y, ratio);
            }
        }
    }
    const float inv = 1.f / scale;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        const int r = it * RPP + tid / LPR;
        if (r >= lo && r < hi) *reinterpret_cast<uint64_t*>(codes + r * DH) = to_e4m3(x[it], inv);
    }
    __syncthreads();   // (every thread has read the old scale)
    if (tid == 0) *ps = scale;
}

// ------------------------------------------------------------------ attention: items of a step
// The query rows of a sequence and key/value head, r = i G + g for new token i and the g-th of the head's G query heads, go
// in blocks of RB.  A block's keys are cut into chunks of c units of UNIT keys, c so that the step's items, (row block,
// chunk) pairs, are at most `items`: with N the sum over the row blocks of their units and X = items - (row blocks),
// c = ceil(N / X) gives at most N / c + (row blocks).  So the long sequences of a batch are cut and the short ones are not,
// whatever their lengths, which the host does not know.  A block of one chunk writes its output, one of several
// partial sums, which k_attn_join adds up in order.
constexpr int UNIT = 128;

struct PagedParams {
    const bf16_t* q;
    bf16_t* o;
    int H, HKV, G;
    float scale_log2;
    int items, spare;      // items per key/value head (the grid), and those beyond one per row block (0: no cuts)
    float* po;             // partial sums of item w, head hk: [w HKV + hk][RB][DH], and their largest score and weight sum
    float2* pml;           // ... [w HKV + hk][RB]
    StepSeqs s;
    Cache c;
};

struct Item {
    int s, tok, n, len;    // sequence, its first new token's row, new tokens, length with them
    int rb, nrb;           // row block, of how many
    int c, chunk, first;   // keys per chunk; chunk of the item; item of the row block's chunk 0 (chunk j: first + j nrb)
    int end;               // keys that the row block's last row sees
};

// The keys that row block rb of a sequence sees: those of its last row.
template <int RB> __device__ __forceinline__ int block_end(const PagedParams& p, int n, int len, int rb) {
    const int i = min((rb * RB + RB - 1) / p.G, n - 1);
    return min(max(len - n + i + 1, 0), p.c.max_pages << p.c.shift);
}

// Item w of a key/value head (BLOCK: row block w instead, chunk 0).  Called by a whole wave; false past the last.
template <int RB, bool BLOCK = false> __device__ __forceinline__ bool find_item(const PagedParams& p, int w, Item& it) {
    const int lane = threadIdx.x & 63, cap = p.c.max_pages << p.c.shift;
    int beg, end, L, nrb, units;   // of sequence base + lane
    auto load = [&](int base, int& at) {
        span64(p.s, base, at, beg, end);
        L = base + lane < p.s.n ? p.s.lens[base + lane] : 0;
        nrb = ((end - beg) * p.G + RB - 1) / RB;
        units = max((min(max(L, 0), cap) + UNIT - 1) / UNIT, 1);
    };
    int at = 0, c = 1 << 23;   // (2^30 keys, the most a table holds)
    if (p.spare > 0) {
        long total = 0;
        for (int base = 0; base < p.s.n; base += 64) {
            load(base, at);
            total += (long)nrb * units;
        }
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) total += __shfl_xor(total, off, 64);
        c = (int)min((total + p.spare - 1) / p.spare, (long)c);
        c = max(__builtin_amdgcn_readfirstlane(c), 1);
    }
    int items = 0, blocks = 0;   // before sequence base
    at = 0;
    for (int base = 0; base < p.s.n; base += 64) {
        if (base > 0 || p.spare == 0 || p.s.n > 64) load(base, at);
        const int cnt = nrb * ((units + c - 1) / c);
        int si = cnt, sb = nrb;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int y = __shfl_up(si, off, 64), z = __shfl_up(sb, off, 64);
            if (lane >= off) { si += y; sb += z; }
        }
        const uint64_t past = __builtin_amdgcn_ballot_w64((BLOCK ? blocks + sb : items + si) > w);
        if (past) {
            const int l = __builtin_ctzll(past);
            it.s = base + l;
            it.tok = __builtin_amdgcn_readlane(beg, l);
            it.n = __builtin_amdgcn_readlane(end, l) - it.tok;
            it.len = __builtin_amdgcn_readlane(L, l);
            it.nrb = __builtin_amdgcn_readlane(nrb, l);
            const int fi = items + __builtin_amdgcn_readlane(si - cnt, l), fb = blocks + __builtin_amdgcn_readlane(sb - nrb, l);
            const int r = BLOCK ? w - fb : w - fi;
            it.rb = r % it.nrb;
            it.chunk = r / it.nrb;
            it.first = fi + it.rb;
            it.c = c * UNIT;
            it.end = block_end<RB>(p, it.n, it.len, it.rb);
            return true;
        }
        items += __builtin_amdgcn_readlane(si, 63);
        blocks += __builtin_amdgcn_readlane(sb, 63);
    }
    return false;
}

// Pages of a walk over a sequence's keys: lane i holds entry i of 64 of its table (and, e4m3, its scales), so that a step
// takes its page without waiting for memory.  Asked for in rising order.
template <bool SCALED> struct PageWalk {
    const int32_t* row;
    int first, id;
    float ks, vs;
    __device__ __forceinline__ void load(const PagedParams& p, int hk, int b) {
        const int lane = threadIdx.x & 63;
        first = b;
        id = b + lane < p.c.max_pages ? row[b + lane] : -1;
        if (id < 0 || id >= p.c.n_pages) id = -1;
        if constexpr (SCALED) {
            const long at = (long)max(id, 0) * p.HKV + hk;
            ks = p.c.ks[at];
            vs = p.c.vs[at];
        }
    }
    __device__ __forceinline__ int page(const PagedParams& p, int hk, int b) {
        if (b - first >= 64) load(p, hk, b);
        return __builtin_amdgcn_readlane(id, b - first);
    }
};

// ------------------------------------------------------------------ k_attn_rows: few rows, many keys
// Attention of blocks of up to 16 rows; bound by the cache's bytes.  A wave takes 32 keys a step, K and V from memory
// straight into its registers, one step ahead of their use, without LDS or barriers; the workgroup's four waves take the
// chunk's steps in turn and add up at the end.
//   S^T = K Q^T: the A operand's row 4 a + b of 16-key half t is key 16 t + 4 b + a, so that a lane's results st[t][e] are
// keys 16 t + 4 e + lg of query l16.
//   O^T = V^T P^T: with contraction element j of lane group lg standing for key 4 j + lg, the weights are the B operand as
// they stand, and lane l16 of the A operand of product n being channel CW l16 + n (CW = DH / 16), it is formed from 8
// loads of CW channels of whole rows (4 rows, 16 lanes each, a load) by a transposition inside the lane.
template <int DH, typename CT> struct RowsStep {
    static constexpr int CW = DH / 16, ESZ = sizeof(CT), NK = DH * ESZ / 64;   // 16-byte K pieces per lane and half
    int4v k[2][NK];
    int v[8][CW * ESZ / 4];
    float ks[2], vs[2];
    bool there[2];   // the half's page
};

__device__ __forceinline__ int fp8_pair(int src, bool high) {   // two e4m3 codes as bf16 (exactly)
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 r = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(src, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(src, 1.f, false);
    return __builtin_bit_cast(int, r);
}

constexpr float LOWEST = -3.402823466e38f;   // a running maximum's start: finite, so that no difference is NaN

template <int DH, typename CT>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_attn_rows(PagedParams p) {
    constexpr int NW = NT / 64, RB = 16, CW = DH / 16, ESZ = sizeof(CT), NKB = DH / 32, NK = DH * ESZ / 64, VD = CW * ESZ / 4;
    constexpr bool E4M3 = ESZ == 1;
    __shared__ float lds_o[NW][RB][DH];
    __shared__ float2 lds_ml[NW][RB];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, lg = lane >> 4;
    const int hk = (int)(blockIdx.x % p.HKV);
    Item it;
    if (!find_item<RB>(p, (int)(blockIdx.x / p.HKV), it)) return;
    const int k0 = it.chunk * it.c, k1 = min(it.end - k0, it.c) + k0;   // the item's keys
    if (it.chunk > 0 && k0 >= it.end) return;
    const int rows = min(it.n * p.G - it.rb * RB, RB);
    const int row = it.rb * RB + l16, qi = row / p.G, h = hk * p.G + row % p.G;
    const int last = it.len - it.n + qi, last0 = it.len - it.n + it.rb * RB / p.G;   // this lane's row, and the block's first
    bf16x8 qf[NKB] = {};
    if (l16 < rows) {
        const bf16_t* src = p.q + ((long)(it.tok + qi) * p.H + h) * DH;
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
            qf[kb] = *reinterpret_cast<const bf16x8*>(src + (E4M3 ? 64 * (kb / 2) + 16 * lg + 8 * (kb % 2) : 32 * kb + 8 * lg));
    }
    floatx4 acc[CW];
#pragma unroll
    for (int n = 0; n < CW; ++n) acc[n] = floatx4{0.f, 0.f, 0.f, 0.f};
    float m = LOWEST, l = 0.f;
    const int koff = (4 * (l16 & 3) + (l16 >> 2)) * DH * ESZ + 16 * lg, voff = lg * DH * ESZ + l16 * CW * ESZ;

    typedef RowsStep<DH, CT> Step;
    PageWalk<E4M3> walk;
    walk.row = p.c.table + (long)it.s * p.c.max_pages;
    if (k1 > k0) walk.load(p, hk, (k0 + 32 * wave) >> p.c.shift);
    auto load = [&](Step& x, int kb) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int key = kb + 16 * t, b = key >> p.c.shift;
            const int id = key < k1 ? walk.page(p, hk, b) : -1;
            x.there[t] = id >= 0;
            if constexpr (E4M3) {
                x.ks[t] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, walk.ks), b - walk.first));
                x.vs[t] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, walk.vs), b - walk.first));
            }
            const long at = ((((long)max(id, 0) * p.HKV + hk) << p.c.shift) + (key & (p.c.page - 1))) * DH * ESZ;
            const uint32_t bytes = id >= 0 ? (uint32_t)min(k1 - key, 16) * DH * ESZ : 0;   // rows past the item's read as zeros
            const auto rk = rsrc((const char*)p.c.k + at, bytes), rv = rsrc((const char*)p.c.v + at, bytes);
#pragma unroll
            for (int i = 0; i < NK; ++i) x.k[t][i] = __builtin_bit_cast(int4v, bload16(rk, koff + 64 * i));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int off = voff + 4 * j * DH * ESZ;
                int(&d)[VD] = x.v[4 * t + j];
                if constexpr (VD == 4) {
                    const int4v y = __builtin_bit_cast(int4v, bload16(rv, off));
                    d[0] = y[0]; d[1] = y[1]; d[2] = y[2]; d[3] = y[3];
                } else if constexpr (VD == 2) {
                    const auto y = __builtin_amdgcn_raw_buffer_load_b64(rv, off, 0, 0);
                    d[0] = y[0]; d[1] = y[1];
                } else {
                    d[0] = __builtin_amdgcn_raw_buffer_load_b32(rv, off, 0, 0);
                }
            }
        }
    };
    auto compute = [&](Step& x, int kb) {
        floatx4 st[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            st[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NKB; ++i) {
                bf16x8 ka;
                if constexpr (E4M3) {
                    const int a = x.k[t][i / 2][2 * (i % 2)], b = x.k[t][i / 2][2 * (i % 2) + 1];
                    ka = __builtin_bit_cast(bf16x8, int4v{fp8_pair(a, false), fp8_pair(a, true), fp8_pair(b, false), fp8_pair(b, true)});
                } else {
                    ka = __builtin_bit_cast(bf16x8, x.k[t][i]);
                }
                st[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qf[i], st[t], 0, 0, 0);
            }
            st[t] *= E4M3 ? x.ks[t] * p.scale_log2 : p.scale_log2;
        }
        const bool masked = kb + 31 > last0 || kb + 32 > k1 || !x.there[0] || !x.there[1];
        if (masked) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = kb + 16 * t + 4 * e + lg;
                    if (key > last || key >= k1 || !x.there[t]) st[t][e] = -INFINITY;
                }
        }
        float bm = fmaxf(fmaxf(fmaxf(st[0][0], st[0][1]), fmaxf(st[0][2], st[0][3])),
                         fmaxf(fmaxf(st[1][0], st[1][1]), fmaxf(st[1][2], st[1][3])));
        // the reference m moves only when a score passes it by more than 8 (weights stay below 2^8)
        if (__builtin_amdgcn_ballot_w64(bm > m + 8.f)) {
            bm = fmaxf(bm, __shfl_xor(bm, 16, 64));
            bm = fmaxf(bm, __shfl_xor(bm, 32, 64));
            const float mn = bm > m + 8.f ? bm : m, a = __builtin_amdgcn_exp2f(m - mn);
#pragma unroll
            for (int n = 0; n < CW; ++n) acc[n] *= a;
            l *= a;
            m = mn;
        }
        floatx4 w[2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[t][e] = __builtin_amdgcn_exp2f(st[t][e] - m);
                l += w[t][e];
            }
        int vb[8][CW / 2];   // bf16 pairs of channels
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < CW / 2; ++i) vb[j][i] = E4M3 ? fp8_pair(x.v[j][i / 2], i % 2) : x.v[j][E4M3 ? 0 : i];
        if (masked && it.n > 1) {
            // A weight of 0 does not hide a value that is not finite (0 x NaN): such values of keys that some rows do not
            // see are taken out here and made NaN in the rows that do.
            bool odd = false;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < CW / 2; ++i)
                    odd = odd || (vb[j][i] & 0x7f800000) == 0x7f800000 || (vb[j][i] & 0x7f80) == 0x7f80;
            if (__builtin_amdgcn_ballot_w64(odd)) {
                floatx4 seen[2];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) seen[t][e] = st[t][e] == -INFINITY ? 0.f : 1.f;
                const bf16x8 sf = pack_bf16(seen[0], seen[1]);
#pragma unroll
                for (int n = 0; n < CW; ++n) {
                    int bad[4];
#pragma unroll
                    for (int jj = 0; jj < 4; ++jj) {
                        bad[jj] = 0;
#pragma unroll
                        for (int z = 0; z < 2; ++z) {
                            const int sh = 16 * (n % 2);
                            int& d = vb[2 * jj + z][n / 2];
                            if (((d >> sh) & 0x7f80) == 0x7f80) {
                                d &= ~(0xffff << sh);
                                bad[jj] |= 0x3f80 << (16 * z);
                            }
                        }
                    }
                    const floatx4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        __builtin_bit_cast(bf16x8, int4v{bad[0], bad[1], bad[2], bad[3]}), sf, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (hit[e] != 0.f) acc[n][e] = __uint_as_float(0x7fc00000u);
                }
            }
        }
        if constexpr (E4M3) {
            w[0] *= x.vs[0];
            w[1] *= x.vs[1];
        }
        const bf16x8 pf = pack_bf16(w[0], w[1]);
#pragma unroll
        for (int n = 0; n < CW; ++n) {
            int4v va;
#pragma unroll
            for (int jj = 0; jj < 4; ++jj)
                va[jj] = __builtin_amdgcn_perm(vb[2 * jj + 1][n / 2], vb[2 * jj][n / 2], n % 2 ? 0x07060302 : 0x05040100);
            acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, va), pf, acc[n], 0, 0, 0);
        }
    };
    Step a, b;
    int kb = k0 + 32 * wave;
    if (kb < k1) load(a, kb);
    while (kb < k1) {
        if (kb + 32 * NW < k1) load(b, kb + 32 * NW);
        compute(a, kb);
        kb += 32 * NW;
        if (kb >= k1) break;
        if (kb + 32 * NW < k1) load(a, kb + 32 * NW);
        compute(b, kb);
        kb += 32 * NW;
    }
    // the four waves' sums: acc[n][e] is channel CW (4 lg + e) + n of query l16
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (lg == 0) lds_ml[wave][l16] = float2{m, l};
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int n = 0; n < CW; ++n) lds_o[wave][l16][CW * (4 * lg + e) + n] = acc[n][e];
    __syncthreads();
    const int r = tid / 16, c0 = (tid % 16) * CW;
    if (r >= rows) return;
    float M = LOWEST, wt[NW], sum = 0.f, o[CW] = {};
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, lds_ml[w][r].x);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        wt[w] = __builtin_amdgcn_exp2f(lds_ml[w][r].x - M);
        sum += wt[w] * lds_ml[w][r].y;
#pragma unroll
        for (int n = 0; n < CW; ++n) o[n] += wt[w] * lds_o[w][r][c0 + n];
    }
    if (it.end <= it.c) {   // the only chunk
        const float inv = sum == 0.f ? 0.f : 1.f / sum;   // no key: zeros
        const int rr = it.rb * RB + r;
        bf16_t* dst = p.o + ((long)(it.tok + rr / p.G) * p.H + hk * p.G + rr % p.G) * DH + c0;
#pragma unroll
        for (int n = 0; n < CW; n += 4)
            *reinterpret_cast<bf16x4*>(dst + n) =
                __builtin_convertvector((floatx4{o[n] * inv, o[n + 1] * inv, o[n + 2] * inv, o[n + 3] * inv}), bf16x4);
    } else {
        const long slot = (long)blockIdx.x * RB + r;
        if (c0 == 0) p.pml[slot] = float2{M, sum};
#pragma unroll
        for (int n = 0; n < CW; n += 4) *reinterpret_cast<floatx4*>(p.po + slot * DH + c0 + n) = floatx4{o[n], o[n + 1], o[n + 2], o[n + 3]};
    }
}

// ------------------------------------------------------------------ k_attn_join
// One wave per row: the sum of its chunks' partial sums, in order (so that the result does not depend on which ended first).
template <int DH, int RB>
__global__ __launch_bounds__(NT) void k_attn_join(PagedParams p, int groups) {   // groups of 4 rows per row block
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int u = blockIdx.x / groups, r = (int)(blockIdx.x % groups) * (NT / 64) + wave, hk = u % p.HKV;
    Item it;
    if (!find_item<RB, true>(p, u / p.HKV, it)) return;
    const int rr = it.rb * RB + r;
    if (it.end <= it.c || rr >= it.n * p.G) return;
    const int chunks = (it.end + it.c - 1) / it.c;
    auto slot = [&](int j) { return ((long)(it.first + j * it.nrb) * p.HKV + hk) * RB + r; };
    float M = LOWEST, sum = 0.f;
    for (int j0 = 0; j0 < chunks; j0 += 64) M = fmaxf(M, j0 + lane < chunks ? p.pml[slot(j0 + lane)].x : LOWEST);
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) M = fmaxf(M, __shfl_xor(M, off, 64));
    constexpr int CPL = DH / 64;   // channels per lane
    float o[CPL] = {};
    for (int j0 = 0; j0 < chunks; j0 += 64) {
        const float2 ml = j0 + lane < chunks ? p.pml[slot(j0 + lane)] : float2{LOWEST, 0.f};
        const float w = __builtin_amdgcn_exp2f(ml.x - M);
        sum += w * ml.y;
        const int many = min(chunks - j0, 64);
#pragma unroll 4
        for (int j = 0; j < many; ++j) {
            const float wj = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), j));
            const float* src = p.po + slot(j0 + j) * DH + CPL * lane;
#pragma unroll
            for (int e = 0; e < CPL; ++e) o[e] += wj * src[e];
        }
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) sum += __shfl_xor(sum, off, 64);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    bf16_t* dst = p.o + ((long)(it.tok + rr / p.G) * p.H + hk * p.G + rr % p.G) * DH + CPL * lane;
#pragma unroll
    for (int e = 0; e < CPL; ++e) dst[e] = from_f<bf16_t>(o[e] * inv);
}
