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

// ------------------------------------------------------------------ k_attn_paged
// One wave per (new token, query head): its keys, 64 / (DH / 8) at a time, each over DH / 8 lanes, with a running softmax
// of its own for every key's place among them (joined at the end).
struct PagedParams {
    const bf16_t* q;
    bf16_t* o;
    long tokens;
    int H, HKV;
    float scale_log2;
    StepSeqs s;
    Cache c;
};

template <int DH, typename CT>
__global__ __launch_bounds__(NT) void k_attn_paged(PagedParams p) {
    constexpr int LPR = DH / 8, KPI = 64 / LPR;
    const int lane = threadIdx.x & 63, c = lane % LPR, kr = lane / LPR;
    const long u = (long)blockIdx.x * (NT / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long tok = u / p.H;
    const int h = (int)(u % p.H), hk = h / (p.H / p.HKV);
    int s, i, n;
    if (tok >= p.tokens || !step_seq(p.s, (int)tok, s, i, n)) return;
    const long keys = min((long)p.s.lens[s] - n + i + 1, (long)p.c.max_pages << p.c.shift);
    float q[8], o[8] = {}, m = -3.402823466e38f, l = 0.f;
    load8(p.q + (tok * p.H + h) * DH + 8 * c, q);
    for (long j0 = 0; j0 < keys; j0 += KPI) {
        const long j = j0 + kr;
        const int id = j < keys ? page_of(p.c, s, j >> p.c.shift) : -1;
        float x = -INFINITY, v[8] = {}, k[8] = {};
        if (id >= 0) {
            const long at = (((long)id * p.HKV + hk) * p.c.page + (j & (p.c.page - 1))) * DH + 8 * c;
            if constexpr (sizeof(CT) == 2) {
                load8((const bf16_t*)p.c.k + at, k);
                load8((const bf16_t*)p.c.v + at, v);
            } else {
                from_e4m3(*(const uint64_t*)((const uint8_t*)p.c.k + at), k);
                from_e4m3(*(const uint64_t*)((const uint8_t*)p.c.v + at), v);
                const float ks = p.c.ks[(long)id * p.HKV + hk], vs = p.c.vs[(long)id * p.HKV + hk];
#pragma unroll
                for (int e = 0; e < 8; ++e) { k[e] *= ks; v[e] *= vs; }
            }
        }
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) dot += q[e] * k[e];
#pragma unroll
        for (int off = 1; off < LPR; off <<= 1) dot += __shfl_xor(dot, off, 64);
        if (id >= 0) x = dot * p.scale_log2;
        const float mn = fmaxf(m, x), a = exp2f(m - mn), w = exp2f(x - mn);
        m = mn;
        l = l * a + w;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = o[e] * a + w * v[e];
    }
    float M = m;
#pragma unroll
    for (int off = LPR; off < 64; off <<= 1) M = fmaxf(M, __shfl_xor(M, off, 64));
    const float a = exp2f(m - M);
    l *= a;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] *= a;
#pragma unroll
    for (int off = LPR; off < 64; off <<= 1) {
        l += __shfl_xor(l, off, 64);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] += __shfl_xor(o[e], off, 64);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;   // no key: zeros
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] *= inv;
    if (kr == 0) store8(p.o + (tok * p.H + h) * DH + 8 * c, o);
}
