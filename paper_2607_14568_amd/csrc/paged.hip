// The attention layers' serving operators (included by gdn.hip): the norm and rotation of a prompt's queries and keys,
// the new tokens' keys and values into a paged cache, and the new tokens' attention over it.
//
// A step brings n new tokens to each sequence; seq_lens[s] counts the tokens of sequence s with them, so that its i-th
// new token stands at position seq_lens[s] - n + i.  Position p lives in page block_table[s][p / page], slot p % page, of
// a cache [n_pages][H_kv][page][d]: the rows of a page and head lie together, page * d elements that one workgroup streams.

// ------------------------------------------------------------------ sequences of a step
struct StepSeqs {
    const int32_t* cu;    // packed: offsets [n + 1] of the new tokens; null: T tokens each
    const int32_t* lens;  // tokens with the new ones [n] (below 0 as 0); null: no cache (positions from 0)
    int n, T;             // sequences; tokens of a dense sequence (packed: of the call)
};

// Inclusive scans over the wave's lanes (values of 0 or more): within rows of 16 lanes, then row ends into the rows behind.
template <typename F> __device__ __forceinline__ int wave_scan(int x, F f) {
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));   // row_shr:1
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));   // row_bcast:15
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));   // row_bcast:31
    return x;
}
__device__ __forceinline__ int scan_add(int x) { return wave_scan(x, [](int a, int b) { return a + b; }); }
__device__ __forceinline__ int scan_max(int x) { return wave_scan(x, [](int a, int b) { return max(a, b); }); }
__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, 63); }
// the lane before's value (lane 0: `first`)
__device__ __forceinline__ int lane_before(int x, int first) {
    return __builtin_amdgcn_update_dpp(first, x, 0x138, 0xf, 0xf, false);   // wave_shr:1
}

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
    end = scan_max(j < q.n ? min(max(q.cu[j + 1], at), q.T) : at);
    beg = lane_before(end, at);
    at = last_lane(end);
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

// cos and sin of pos * freq[i]: the angle in float64 (a float32 product is off by 2^-24 of an angle of up to 10^5 radians), in
// turns, reduced to a quadrant n and the rest f in [-1/2, 1/2] quarter turns, whose sine and cosine are polynomials in f^2
// (fitted for the least largest error at those degrees and rounded to float: off by 2^-28.1 and 2^-27.1, in float steps by
// 2^-24.5 and 2^-24.0).  With f rounded to float off by at most 2^-23.6 of 1 and 2^-26 on average, less than sincospif of the
// rounded half turns (2^-23.1, 2^-25.3), and no slower.  (The sine unit takes turns and is off by 2^-22.9.)
__device__ __forceinline__ double turns(const Turn& t, int i) { return t.freq[i] * 0.15915494309189535; }   // per position
__device__ __forceinline__ void angle(double turns, double pos, float& cs, float& sn) {
    double a = pos * turns;
    a = 4. * (a - rint(a));
    const float n = rintf((float)a), f = (float)(a - (double)n), u = f * f;
    float s = -0.004602177068591118f, c = 0.0009036316769197583f;
    s = __builtin_fmaf(s, u, 0.07968022674322128f);
    s = __builtin_fmaf(s, u, -0.6459634900093079f);
    s = __builtin_fmaf(s, u, -4.371139e-8f);   // pi / 2 - 1.57079637
    s = __builtin_fmaf(f, 1.57079637f, f * s);
    c = __builtin_fmaf(c, u, -0.02086007222533226f);
    c = __builtin_fmaf(c, u, 0.25366920232772827f);
    c = __builtin_fmaf(c, u, -1.2337005138397217f);
    c = __builtin_fmaf(c, u, 1.f);
    const int k = (int)n;   // -2 .. 2
    sn = k & 1 ? c : s;
    cs = k & 1 ? s : c;
    sn = k & 2 ? -sn : sn;
    cs = (k + 1) & 2 ? -cs : cs;
}

// cos and sin of the pairs of a chunk's 8 channels, from tables [rot / 2] of a position; the sign of the sine is that of the
// channel's own term: y = x cos + partner sin.
__device__ __forceinline__ void angles(const Turn& t, int c, const float* tc, const float* ts, float (&cs)[8], float (&sn)[8]) {
    if (8 * c >= t.rot) {
#pragma unroll
        for (int e = 0; e < 8; ++e) { cs[e] = 1.f; sn[e] = 0.f; }
    } else if (t.near) {
        const floatx4 a = f4(tc + 4 * c), b = f4(ts + 4 * c);
#pragma unroll
        for (int e = 0; e < 8; ++e) { cs[e] = a[e / 2]; sn[e] = e % 2 ? b[e / 2] : -b[e / 2]; }
    } else {
        const int hc = t.rot / 16, first = c < hc, at = 8 * (first ? c : c - hc);
        const floatx4 a = f4(tc + at), a2 = f4(tc + at + 4), b = f4(ts + at), b2 = f4(ts + at + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            cs[e] = e < 4 ? a[e] : a2[e - 4];
            sn[e] = e < 4 ? b[e] : b2[e - 4];
            if (first) sn[e] = -sn[e];
        }
    }
}

// x from another lane of the 16 of its DPP row
template <int CTRL> __device__ __forceinline__ float dpp(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
constexpr int XOR1 = 0xb1, XOR2 = 0x4e, REVERSE4 = 0x1b, MIRROR8 = 0x141, MIRROR16 = 0x140, ROTATE8 = 0x128;
// sums and maxima over LPR = 8 or 16 neighbouring lanes, in each of them
template <int LPR, typename F> __device__ __forceinline__ float over_row(float x, F f) {
    x = f(x, dpp<XOR1>(x));
    x = f(x, dpp<XOR2>(x));
    x = f(x, dpp<MIRROR8>(x));
    if constexpr (LPR == 16) x = f(x, dpp<MIRROR16>(x));
    return x;
}

// x: this lane's 8 channels; w: their weights or null; cs, sn: from angles() (used when t.freq).  y = x w / sqrt(mean(x^2)
// + eps), then (a, b) -> (a cos - b sin, b cos + a sin) over the pairs: every channel is x cs + partner sn.  (Lanes exchange
// through DPP; by ds_bpermute a prompt of 4133 tokens took 18.4 us into an e4m3 cache, 17.2 so.)
template <int DH>
__device__ __forceinline__ void turn_row(const Turn& t, bool norm, const float* w, const float (&cs)[8], const float (&sn)[8], float (&x)[8]) {
    constexpr int LPR = DH / 8;
    const int lane = threadIdx.x & 63, c = lane % LPR;
    if (norm) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += x[e] * x[e];
        ss = over_row<LPR>(ss, [](float a, float b) { return a + b; });
        const floatx4 w0 = f4(w + 8 * c), w1 = f4(w + 8 * c + 4);
        const float var = ss * (1.f / DH) + t.eps;
        float r = __builtin_amdgcn_rsqf(var);   // (off by 2^-23 at most; 1 / sqrtf takes some 25 instructions)
        if (__builtin_amdgcn_ballot_w64(var < 0x1p-126f)) r = var < 0x1p-126f ? 1.f / sqrtf(var) : r;   // (it takes those as 0)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= r * (e < 4 ? w0[e] : w1[e - 4]);
    }
    if (t.freq) {
        const int hc = t.rot / 16;   // partners are hc lanes apart
        float y[8];
        if (t.near) {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = x[e ^ 1];
        } else if (LPR == 16 && hc == 8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = dpp<ROTATE8>(x[e]);
        } else if (hc == 4) {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = dpp<REVERSE4>(dpp<MIRROR8>(x[e]));
        } else {
            const int from = c < hc ? lane + hc : c < 2 * hc ? lane - hc : lane;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = __shfl(x[e], from, 64);
        }
        if (8 * c >= t.rot) {   // (no partner: nothing of another channel, not even 0 times it)
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * cs[e] + y[e] * sn[e];
    }
}

// 8 channels as they lie in memory
template <typename IO> struct Chunk8;
template <> struct Chunk8<bf16_t> {
    short8 v;
    __device__ __forceinline__ void load(const bf16_t* p) { v = *reinterpret_cast<const short8*>(p); }
    __device__ __forceinline__ void zero() { v = short8{}; }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = bf(v[e]);
    }
};
template <> struct Chunk8<float> {
    floatx4 a, b;
    __device__ __forceinline__ void load(const float* p) { a = f4(p); b = f4(p + 4); }
    __device__ __forceinline__ void zero() { a = b = floatx4{}; }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[4 + e] = b[e]; }
    }
};
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

constexpr float LOWEST = -3.402823466e38f;   // a running maximum's start: finite, so that no difference is NaN

// ------------------------------------------------------------------ e4m3
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
    for (int e = 0; e < 8; ++e) y[e] = fabsf(x[e]) <= -LOWEST ? x[e] * inv : __uint_as_float(0x7fc00000u);
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

// This lane's 8 codes of rows r0, r0 + step, .. below r1 brought to another scale (N rows' loads at a time).  (A single token
// past its page's scale: 256 sequences, all their pages of 64, K and V of 8 heads, 3.5 us more than a step that keeps them.)
template <int N> __device__ __forceinline__ void rescale(uint8_t* codes, int pitch, int r0, int r1, int step, float ratio) {
#pragma unroll 1
    for (int r = r0; r < r1; r += N * step) {
        uint64_t y[N];
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (r + i * step < r1) y[i] = *reinterpret_cast<const uint64_t*>(codes + (r + i * step) * pitch);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (r + i * step < r1) {
                float z[8];
                from_e4m3(y[i], z);
                *reinterpret_cast<uint64_t*>(codes + (r + i * step) * pitch) = to_e4m3(z, ratio);
            }
    }
}

// ------------------------------------------------------------------ k_rows: tokens' rows, normed and rotated
// One wave takes `per` groups of 64 / (DH / 8) rows of one token: its q heads, its k heads and, into a cache, its v heads
// (those as they are); into an e4m3 cache only where a sequence has one new token, whose rows are then all there is of a
// page's and head's new values.  Each lane forms one angle of the token's position, the wave's tables of them lie in LDS.
// Bound by memory: every row is read once and written once, a lane's 16 bytes (8 channels) an access, so that a head's row
// lies in 8 or 16 neighbouring lanes and its norm is a sum over them by DPP.  Measured: q and k of 10240 tokens, 24 heads of
// 128, 27.6 us (4.6 TB/s, a copy reaches 5.2; 25.0 without norm and rotation); q, k and v of 11245 tokens, 32 heads, into a
// bf16 cache 41 us (4.5 TB/s); one sequence's token 4.2 us.  Rows of two groups are loaded before the first is used; of eight
// it was slower (30.3 us against 25.9 with the inputs in the last-level cache).
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

struct __attribute__((aligned(16))) RowTables { float c[64], s[64], qw[128], kw[128]; };   // a wave's angles and weights

template <typename IO, int DH, bool E4M3, bool QONLY = false>
__device__ __forceinline__ void token_rows(const RowsParams& p, int wave, RowTables& tab) {
    constexpr int LPR = DH / 8, RPG = 64 / LPR, AHEAD = 2;
    const int token = wave / p.units, unit = wave - token * p.units, lane = threadIdx.x & 63, c = lane % LPR;
    if (token >= p.tokens) return;
    const long tok = token;
    int s = 0, i = 0, n = 0;
    if (!step_seq(p.s, token, s, i, n)) return;
    const int pos = p.pos ? p.pos[tok] : p.s.lens ? max(p.s.lens[s], 0) - n + i : i;
    // The weights lie in LDS: read for each row through the CU's cache, twice a bf16 row's bytes, they cost 1.1 us more of 28.
    if (p.qw && 2 * lane < DH)
#pragma unroll
        for (int e = 0; e < 2; ++e) tab.qw[2 * lane + e] = p.qw[2 * lane + e];
    if (!QONLY && p.kw && 2 * lane < DH)
#pragma unroll
        for (int e = 0; e < 2; ++e) tab.kw[2 * lane + e] = p.kw[2 * lane + e];
    __builtin_amdgcn_wave_barrier();
    float cs[8], sn[8];
    if (p.t.freq) {
        if (lane < p.t.rot / 2) angle(turns(p.t, lane), pos, tab.c[lane], tab.s[lane]);
        __builtin_amdgcn_wave_barrier();   // (the wave's LDS accesses stay in order)
        angles(p.t, c, tab.c, tab.s, cs, sn);
    }
    const int HQ = p.q ? p.H : 0, rows = QONLY ? p.H : HQ + p.HKV + (p.v ? p.HKV : 0);
    const int id = !QONLY && !p.ko && pos >= 0 ? page_of(p.c, s, pos >> p.c.shift) : -1;
    const int slot = pos & (p.c.page - 1);
    // AHEAD groups' rows are loaded before the first is used
    for (int g0 = 0; g0 < p.per; g0 += AHEAD) {
        Chunk8<IO> in[AHEAD];
#pragma unroll
        for (int z = 0; z < AHEAD; ++z) {
            const int j = (unit * p.per + g0 + z) * RPG + lane / LPR;
            const IO* src = QONLY || j < HQ ? (const IO*)p.q + tok * p.qs + j * DH
                            : j < HQ + p.HKV ? (const IO*)p.k + tok * p.ks + (j - HQ) * DH
                                             : (const IO*)p.v + tok * p.vs + (j - HQ - p.HKV) * DH;
            in[z].zero();
            if (g0 + z < p.per && j < rows) in[z].load(src + 8 * c);
        }
#pragma unroll
        for (int z = 0; z < AHEAD; ++z) {
            const int j = (unit * p.per + g0 + z) * RPG + lane / LPR;
            const int kind = QONLY || j < HQ ? 0 : j < HQ + p.HKV ? 1 : 2;   // q, k, v
            const int h = kind == 0 ? j : kind == 1 ? j - HQ : j - HQ - p.HKV;
            if (g0 + z >= p.per) break;
            float x[8];
            in[z].get(x);
            // (a row's lanes share their kind, and the exchanges stay inside a row)
            if (kind < 2) turn_row<DH>(p.t, (kind == 0 ? p.qw : p.kw) != nullptr, kind == 0 ? tab.qw : tab.kw, cs, sn, x);
            if (j >= rows) continue;
            if (kind == 0) {
                store8((IO*)p.qo + (tok * p.H + h) * DH + 8 * c, x);
            } else if (p.ko) {
                store8((IO*)p.ko + (tok * p.HKV + h) * DH + 8 * c, x);
            } else if (id >= 0) {
                const long at = (((long)id * p.HKV + h) << p.c.shift) * DH + 8 * c;   // of slot 0
                if constexpr (!E4M3) {
                    store8((IO*)(kind == 1 ? p.c.k : p.c.v) + at + slot * DH, x);
                } else {
                    float amax = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[e]) <= -LOWEST ? fabsf(x[e]) : 0.f);
                    amax = over_row<LPR>(amax, [](float a, float b) { return fmaxf(a, b); });
                    uint8_t* codes = (uint8_t*)(kind == 1 ? p.c.k : p.c.v) + at;
                    float* ps = (kind == 1 ? p.c.ks : p.c.vs) + (long)id * p.HKV + h;
                    float scale = power_scale(amax);
                    if (slot > 0) {
                        const float old = *ps;
                        if (old >= scale) {
                            scale = old;
                        } else {
                            rescale<4>(codes, DH, 0, slot, 1, old / scale);
                        }
                    }
                    *reinterpret_cast<uint64_t*>(codes + slot * DH) = to_e4m3(x, 1.f / scale);
                    if (c == 0) *ps = scale;
                }
            }
        }
    }
}

template <typename IO, int DH, bool E4M3>
__global__ __launch_bounds__(NT) void k_rows(RowsParams p) {
    __shared__ RowTables tab[NT / 64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    token_rows<IO, DH, E4M3>(p, (int)blockIdx.x * (NT / 64) + wave, tab[wave]);
}

// ------------------------------------------------------------------ k_append_e4m3
// The block-th page that the step's new tokens touch (dense: of `each` pages that a sequence can touch): its sequence s,
// the page's index b in it, the positions [first, len) of the sequence's new tokens and the call's row of the first of
// them.  Called by a whole wave; false where there is none.
__device__ __forceinline__ bool touched_block(const StepSeqs& q, int shift, int each, int block, int& s, int& b, int& first, int& len,
                                              int& row) {
    if (!q.cu) {
        s = block / each;
        len = max(tab(q.lens, s), 0);
        first = max(len - q.T, 0);   // (a token before position 0 is not written)
        b = (first >> shift) + block % each;
        row = s * q.T + q.T - (len - first);
        return len > 0 && b <= (len - 1) >> shift;
    }
    const int lane = threadIdx.x & 63;
    int at = 0, beg, end, before = 0;
    for (int base = 0; base < q.n; base += 64) {
        span64(q, base, at, beg, end);
        const int L = base + lane < q.n ? max(q.lens[base + lane], 0) : 0;
        const int f = max(L - (end - beg), 0);
        const int cnt = end > beg && L > 0 ? ((L - 1) >> shift) - (f >> shift) + 1 : 0;
        const int sum = scan_add(cnt);
        const uint64_t past = __builtin_amdgcn_ballot_w64(before + sum > block);
        if (past) {
            const int l = __builtin_ctzll(past);
            s = base + l;
            first = __builtin_amdgcn_readlane(f, l);
            len = __builtin_amdgcn_readlane(L, l);
            b = (first >> shift) + block - before - __builtin_amdgcn_readlane(sum - cnt, l);
            row = __builtin_amdgcn_readlane(end, l) - (len - first);
            return true;
        }
        before += last_lane(sum);
    }
    return false;
}

// One workgroup per (touched page, head, K or V), `page_wgs` in all, ahead of those of the q rows.  It holds the page's new
// tokens in registers, finds their largest value, and writes codes and scale.  The angle of slot r = RPP it + i of the page
// at position a is that of a + RPP it and that of i added up, a product of two table entries: (RPP + IT) rot / 2 sines
// for RPP IT rows.  A scale needs its page's and head's largest value before the first code is written, so the unit of work
// is the page: in registers the values are read once and only codes (half the bytes) are written.
// Bound by the norm's and the angles' arithmetic: 4133 tokens of a prompt, 32 heads of 128, 15.9 us (3.7 TB/s over q, k, v
// and the codes); without norm and rotation 11.8 us.  With the q rows' workgroups in between the pages' it was 23.6
// against 18.4 us: the pages, the longer units, have to start first.
template <int DH, int IT>   // IT: passes of NT / (DH / 8) rows over a page
__global__ __launch_bounds__(NT) void k_append_e4m3(RowsParams p, int page_wgs, int each) {
    constexpr int LPR = DH / 8, RPP = NT / LPR, NP = DH / 2;
    __shared__ float red[NT / 64];
    __shared__ __align__(16) float tables[2][RPP + IT][NP], kw[DH];
    auto &tc = tables[0], &ts = tables[1];   // of i, then of a + RPP it
    const int tid = threadIdx.x, c = tid % LPR, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if ((int)blockIdx.x >= page_wgs) {
        static_assert(sizeof(RowTables) * (NT / 64) <= sizeof tables, "the tables of the q rows' waves");
        token_rows<bf16_t, DH, false, true>(p, ((int)blockIdx.x - page_wgs) * (NT / 64) + wave, reinterpret_cast<RowTables*>(tables)[wave]);
        return;
    }
    const int u = (int)blockIdx.x;
    const int is_v = u & 1, h = u / 2 % p.HKV;   // (a page's K and V of all heads side by side)
    int s, b, first, len, row;
    if (!touched_block(p.s, p.c.shift, each, u / 2 / p.HKV, s, b, first, len, row)) return;
    const int id = __builtin_amdgcn_readfirstlane(page_of(p.c, s, b));
    if (id < 0) return;
    const int at0 = b << p.c.shift;   // position of the page's first slot (b lies in the table: under 2^30)
    const int lo = max(first - at0, 0), hi = min(len - at0, p.c.page);   // its new slots
    const bf16_t* src = (const bf16_t*)(is_v ? p.v : p.k) + h * DH + 8 * c;
    const long stride = is_v ? p.vs : p.ks;
    Chunk8<bf16_t> in[IT];
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        const int r = it * RPP + tid / LPR;
        in[it].zero();
        if (r >= lo && r < hi) in[it].load(src + (row + (at0 + r - first)) * stride);
    }
    float x[IT][8], amax = 0.f;
    if (!is_v) {
        if (p.kw && tid < DH) kw[tid] = p.kw[tid];
        const int np = p.t.rot / 2;
        const int j = tid % NP;
        if (j < np) {
            const double f = turns(p.t, j);
#pragma unroll
            for (int i = 0; i < RPP + IT; i += NT / NP) {
                const int r = i + tid / NP;
                if (r < RPP + IT) angle(f, r < RPP ? r : at0 + (r - RPP) * RPP, tc[r][j], ts[r][j]);
            }
        }
        __syncthreads();
        float cs[8], sn[8];
        if (np) angles(p.t, c, tc[tid / LPR], ts[tid / LPR], cs, sn);
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            in[it].get(x[it]);
            if (it * RPP >= hi || (it + 1) * RPP <= lo) continue;   // (the whole workgroup's)
            float ca[8], sa[8], ct[8], st[8];
            if (np) {
                angles(p.t, c, tc[RPP + it], ts[RPP + it], ca, sa);
                // both sines carry the channel's sign g: (g s)(g s') = s s' and g (s c' + c s') as wanted
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    ct[e] = cs[e] * ca[e] - sn[e] * sa[e];
                    st[e] = sn[e] * ca[e] + cs[e] * sa[e];
                }
            }
            turn_row<DH>(p.t, p.kw != nullptr, kw, ct, st, x[it]);
        }
    } else {
#pragma unroll
        for (int it = 0; it < IT; ++it) in[it].get(x[it]);
    }
#pragma unroll
    for (int it = 0; it < IT; ++it)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float m = fabsf(x[it][e]);
            amax = fmaxf(amax, m <= -LOWEST ? m : 0.f);
        }
    amax = __builtin_bit_cast(float, last_lane(scan_max(__builtin_bit_cast(int, amax))));   // (0 or more: in order as integers)
    if ((tid & 63) == 0) red[wave] = amax;
    __syncthreads();
    amax = red[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) amax = fmaxf(amax, red[w]);
    float scale = power_scale(amax);
    float* ps = (is_v ? p.c.vs : p.c.ks) + (long)id * p.HKV + h;
    uint8_t* codes = (uint8_t*)(is_v ? p.c.v : p.c.k) + (((long)id * p.HKV + h) << p.c.shift) * DH + 8 * c;
    if (lo > 0) {   // the page holds earlier tokens of the sequence, in its old scale
        const float old = *ps;
        if (old >= scale) {
            scale = old;
        } else {
            rescale<4>(codes, DH, tid / LPR, lo, RPP, old / scale);
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
// in blocks of RB.  A block's keys are cut into chunks of c units of UNIT keys, c from the step's lengths, which the host
// does not know: the least with which all items, (row block, chunk) pairs, are resident at once (`round` of them per
// key/value head); where that is more than `fine` units and the lengths leave a fifth of them idle, max(fine, N / spare)
// with N the units of all row blocks, which gives at most N / c + (row blocks) items.  So the long sequences of a batch are
// cut and the short ones are not.  A block of one chunk writes its output, one of several partial sums, which k_attn_join
// adds up in order.
// Scores, maxima, weight sums and outputs are fp32.  The matrix instruction with the values takes the weights as bf16: two
// numbers each in k_attn_rows, where its products are nearly free (off by 2^-15; the outputs' error against 64 bits is that of
// their own rounding, 0.0017), one in k_attn_tile, which such products bound (off by 2^-8 of each at most, up and down over the
// keys: error 0.0023; with two numbers each 222 us against 168 for the piece below).
constexpr int UNIT = 128;

// x / d for 0 <= x < 2^31 by one product: m = ceil(2^sh / d), sh = 31 + ceil(log2 d); m d - 2^sh < d <= 2^(sh - 31), so that x
// times it stays below 2^sh.
struct Div { uint32_t m, sh; };
__device__ __forceinline__ int div_by(int x, Div d) { return (int)(((uint64_t)(uint32_t)x * d.m) >> d.sh); }
// ceil(x / c) for 0 <= x < 2^24, 1 <= c: the quotient by a reciprocal is off by less than one
__device__ __forceinline__ int ceil_div(int x, int c, float rc) {
    int q = (int)((float)x * rc);
    q += (long)q * c < x;
    q += (long)q * c < x;
    return q - ((long)(q - 1) * c >= x && q > 0);
}

struct PagedParams {
    const bf16_t* q;
    bf16_t* o;
    int H, HKV, G;
    Div by_hkv, by_g;
    float scale_log2;
    int round, fine, spare; // see above; spare 0: no cuts
    float* po;             // partial sums of item w, head hk: [w HKV + hk][RB][DH], and their largest score and weight sum
    float2* pml;           // ... [w HKV + hk][RB]
    StepSeqs s;
    Cache c;
};

struct Item {
    int s, tok, n, len;    // sequence, its first new token's row, new tokens, length with them
    int rb, nrb;           // row block, of how many
    int c, chunks, chunk, first;   // keys per chunk, chunks, chunk of the item; the sequence's first item (see item_of)
    int end;               // keys that the row block's last row sees
};

// Item of chunk j of the row block: chunk by chunk, even ones from the block with the most keys down, odd ones up, so that
// two items a CU have about the same keys together.
__device__ __forceinline__ int item_of(const Item& it, int j) {
    return it.first + j * it.nrb + (j % 2 ? it.rb : it.nrb - 1 - it.rb);
}

// The keys that row block rb of a sequence sees: those of its last row.
template <int RB> __device__ __forceinline__ int block_end(const PagedParams& p, int n, int len, int rb) {
    const int i = min(div_by(rb * RB + RB - 1, p.by_g), n - 1);
    return min(max(len - n + i + 1, 0), p.c.max_pages << p.c.shift);
}

// Item w of a key/value head (BLOCK: row block w instead, chunk 0).  Called by a whole wave; false past the last.
template <int RB, bool BLOCK = false> __device__ __forceinline__ bool find_item(const PagedParams& p, int w, Item& it) {
    const int lane = threadIdx.x & 63, cap = p.c.max_pages << p.c.shift;
    int beg, end, L, nrb, units;   // of sequence base + lane
    auto load = [&](int base, int& at) {
        span64(p.s, base, at, beg, end);
        L = base + lane < p.s.n ? max(p.s.lens[base + lane], 0) : 0;
        nrb = ((end - beg) * p.G + RB - 1) / RB;
        units = max((min(L, cap) + UNIT - 1) / UNIT, 1);
    };
    int at = 0, c = 1 << 23;   // (2^30 keys, the most a table holds)
    if (p.spare > 0) {
        // the sum over the row blocks of ceil(units / c) (a lane's share held to 2^24: what matters is whether it is small)
        auto count = [&](int c) {
            const float rc = 1.f / (float)c;
            int sum = 0, at = 0;
            for (int base = 0; base < p.s.n; base += 64) {
                if (base > 0 || p.s.n > 64) load(base, at);
                sum = (int)min((long)nrb * ceil_div(units, c, rc) + sum, 1L << 24);
            }
            return last_lane(scan_add(sum));
        };
        load(0, at);
        // N as a float, 2^-20 off at most, which the divisions below make up for
        float total = 0.f;
        for (int base = 0, z = 0; base < p.s.n; base += 64) {
            if (base > 0 || p.s.n > 64) load(base, z);
            total += (float)nrb * (float)units;
        }
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) total += __shfl_xor(total, off, 64);
        total *= 1.f - 0x1p-19f;
        c = max((int)min(ceilf(total / (float)p.round), 0x1p23f), RB == 16 ? 1 : 4);   // (a tile's chunk of fewer keys is mostly joining)
        auto uneven = [&](int c) { return c > p.fine && total < 0.8f * (float)c * (float)p.round; };
        bool fits;
        for (;;) {
            fits = count(c) <= p.round;
            if (fits || c >= 1 << 23 || uneven(c)) break;
            c += (c + 7) / 8;
        }
        if (!fits || uneven(c)) c = max((int)min(ceilf(total * (1.f + 0x1p-17f) / (float)p.spare), 0x1p23f), p.fine);
        c = min(c, 1 << 23);
        c = __builtin_amdgcn_readfirstlane(c);
    }
    int items = 0, blocks = 0;   // before sequence base
    at = 0;
    for (int base = 0; base < p.s.n; base += 64) {
        if (base > 0 || p.spare == 0 || p.s.n > 64) load(base, at);
        const int cnt = nrb * ceil_div(units, c, 1.f / (float)c);
        const int si = scan_add(cnt), sb = BLOCK ? scan_add(nrb) : 0;
        const uint64_t past = __builtin_amdgcn_ballot_w64((BLOCK ? blocks + sb : items + si) > w);
        if (past) {
            const int l = __builtin_ctzll(past);
            it.s = base + l;
            it.tok = __builtin_amdgcn_readlane(beg, l);
            it.n = __builtin_amdgcn_readlane(end, l) - it.tok;
            it.len = __builtin_amdgcn_readlane(L, l);
            it.nrb = __builtin_amdgcn_readlane(nrb, l);
            const int fi = items + __builtin_amdgcn_readlane(si - cnt, l);
            const int r = w - (BLOCK ? blocks + __builtin_amdgcn_readlane(sb - nrb, l) : fi);
            int z = 0;
            it.chunk = r;
            if (it.nrb > 1) {
                it.chunk = r / it.nrb;
                z = r - it.chunk * it.nrb;
            }
            it.rb = it.chunk % 2 ? z : it.nrb - 1 - z;   // see item_of
            it.first = fi;
            it.end = block_end<RB>(p, it.n, it.len, it.rb);
            it.chunks = 1;
            it.c = max(it.end, 1);
            if (it.end > c * UNIT) {   // as many chunks as chunks of c units make, all of one size
                it.chunks = (it.end + c * UNIT - 1) / (c * UNIT);
                it.c = ((it.end + it.chunks - 1) / it.chunks + UNIT - 1) / UNIT * UNIT;
                it.chunks = (it.end + it.c - 1) / it.c;
            }
            return true;
        }
        items += last_lane(si);
        blocks += last_lane(sb);
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
            ks = vs = 1.f;
            if (id >= 0) {
                ks = p.c.ks[(long)id * p.HKV + hk];
                vs = p.c.vs[(long)id * p.HKV + hk];
            }
        }
    }
    __device__ __forceinline__ void reach(const PagedParams& p, int hk, int b, int b_last) {   // up to 64 pages b .. b_last
        if (b_last - first >= 64) load(p, hk, b);
    }
    __device__ __forceinline__ int page(int b) const { return __builtin_amdgcn_readlane(id, b - first); }
    __device__ __forceinline__ float kscale(int b) const { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, ks), b - first)); }
    __device__ __forceinline__ float vscale(int b) const { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, vs), b - first)); }
};

// Eight e4m3 codes times their scale as bf16: exact for a power of two, which is what gdn_kv_append makes a scale (the
// instruction multiplies by the scale's exponent alone, so it must be a positive normal number); any other one's products are
// rounded to bf16, as keys and values that were cached in bf16 are.
__device__ __forceinline__ int4v fp8_scaled(int a, int b, float scale) {
    if ((__float_as_uint(scale) & 0x7fffff) == 0 && __float_as_uint(scale) - 0x800000u < 0x7f000000u)
        return int4v{__builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false)),
                     __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true)),
                     __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false)),
                     __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true))};
    float x[8];
    from_e4m3((uint64_t)(uint32_t)a | (uint64_t)(uint32_t)b << 32, x);
    return __builtin_bit_cast(int4v, pack_bf16(floatx4{x[0], x[1], x[2], x[3]} * scale, floatx4{x[4], x[5], x[6], x[7]} * scale));
}

// c + the eight values
__device__ __forceinline__ float sum_bf16(bf16x8 w, float c) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef float floatx2 __attribute__((ext_vector_type(2)));
    const bf16x2 one = __builtin_convertvector((floatx2{1.f, 1.f}), bf16x2);
#pragma unroll
    for (int i = 0; i < 8; i += 2) c = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{w[i], w[i + 1]}, one, c, false);
    return c;
}

// Eight weights as two bf16 numbers each, hi + lo, off by 2^-15 of them at most: hi the upper half of the float's bits, lo
// what is left, under 2^-7 of it, rounded.  2^-20 of the weight more keeps lo's sign that of hi where nothing is left, so that an
// infinite value's products with both add up to that infinity (0 x infinity and a difference of infinities are NaN).
__device__ __forceinline__ void split_weights(floatx4 a, floatx4 b, bf16x8& hi, bf16x8& lo) {
    int4v h;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float x = i < 2 ? a[2 * i] : b[2 * i - 4], y = i < 2 ? a[2 * i + 1] : b[2 * i - 3];
        h[i] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302);
    }
    auto rest = [](float w) { return __builtin_fmaf(w, 1.f + 0x1p-20f, -__uint_as_float(__float_as_uint(w) & 0xffff0000u)); };
    hi = __builtin_bit_cast(bf16x8, h);
    lo = pack_bf16(floatx4{rest(a[0]), rest(a[1]), rest(a[2]), rest(a[3])}, floatx4{rest(b[0]), rest(b[1]), rest(b[2]), rest(b[3])});
}

// ------------------------------------------------------------------ k_attn_rows: few rows, many keys
// Attention of blocks of up to 16 rows; bound by the cache's bytes.  A wave takes 32 keys a step, K and V from memory
// straight into its registers, 16 KB of steps ahead of their use, without LDS or barriers; the workgroup's waves take the
// chunk's steps in turn and add up at the end.  Two workgroups per CU (256 registers a wave) keep 128 KB of loads in
// flight on a CU; matrix products are nearly free beside them, and a row block of up to 16 rows costs no more than one row.
// Measured: a token of 64 sequences of 526 to 8138 keys, 695 MB of bf16 cache in 125 us (5.6 TB/s; reads alone reach 6.4); the
// same in e4m3 74 us (4.7 TB/s); one sequence of 131072 keys 94 us (5.7 TB/s).  With few items what bounds it is the load path
// of a CU: 776 keys of one sequence, 8 workgroups, 1 us per 128 keys, since a K operand's load touches 64 bytes of 16 rows, a
// third of that path's rate; eight waves a workgroup there gained nothing.
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

// One row over keys k0 .. k1 - 1 by one wave without the matrix units: 64 / (DH / 8) keys at a time, each over DH / 8 lanes,
// with a running softmax for each place among them.  o: this lane's 8 channels, the same in all places; m, l of the row.
template <int DH, typename CT>
__device__ __forceinline__ void plain_row(const PagedParams& p, const Item& it, int hk, int row, int k0, int k1, float& m, float& l,
                                          float (&o)[8]) {
    constexpr int LPR = DH / 8, KPI = 64 / LPR;
    const int lane = threadIdx.x & 63, c = lane % LPR, qi = div_by(row, p.by_g);
    const int last = it.len - it.n + qi;
    float q[8];
    Chunk8<bf16_t> y;
    y.load(p.q + ((long)(it.tok + qi) * p.H + hk * p.G + row - qi * p.G) * DH + 8 * c);
    y.get(q);
    m = LOWEST;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.f;
#pragma unroll 1
    for (int j = k0 + lane / LPR; j - lane / LPR <= min(last, k1 - 1); j += KPI) {
        const int id = j <= min(last, k1 - 1) ? page_of(p.c, it.s, j >> p.c.shift) : -1;
        float dot = 0.f, v[8] = {}, ks = 1.f, vs = 1.f;
        if (id >= 0) {
            const long at = ((((long)id * p.HKV + hk) << p.c.shift) + (j & (p.c.page - 1))) * DH + 8 * c;
            float k[8];
            if constexpr (sizeof(CT) == 2) {
                y.load((const bf16_t*)p.c.k + at);
                y.get(k);
                y.load((const bf16_t*)p.c.v + at);
                y.get(v);
            } else {
                from_e4m3(*(const uint64_t*)((const uint8_t*)p.c.k + at), k);
                from_e4m3(*(const uint64_t*)((const uint8_t*)p.c.v + at), v);
                ks = p.c.ks[(long)id * p.HKV + hk];
                vs = p.c.vs[(long)id * p.HKV + hk];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) dot += q[e] * k[e];
        }
#pragma unroll
        for (int off = 1; off < LPR; off <<= 1) dot += __shfl_xor(dot, off, 64);
        const float x = id >= 0 ? dot * (ks * p.scale_log2) : -INFINITY;
        const float mn = fmaxf(m, x), a = __builtin_amdgcn_exp2f(m - mn), w = __builtin_amdgcn_exp2f(x - mn);
        m = mn;
        l = l * a + w;
        if (id >= 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = o[e] * a + w * vs * v[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] *= a;
        }
    }
    float M = m;
#pragma unroll
    for (int off = LPR; off < 64; off <<= 1) M = fmaxf(M, __shfl_xor(M, off, 64));
    const float a = __builtin_amdgcn_exp2f(m - M);
    m = M;
    l *= a;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] *= a;
#pragma unroll
    for (int off = LPR; off < 64; off <<= 1) {
        l += __shfl_xor(l, off, 64);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] += __shfl_xor(o[e], off, 64);
    }
}

template <int DH, typename CT>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_attn_rows(PagedParams p) {
    constexpr int NW = NT / 64, RB = 16, CW = DH / 16, ESZ = sizeof(CT), NKB = DH / 32, NK = DH * ESZ / 64, VD = CW * ESZ / 4;
    constexpr bool E4M3 = ESZ == 1;
    __shared__ __align__(16) float lds_o[NW][RB][DH + 4];   // (rows 4 banks apart: 16 rows' 16-byte accesses meet no bank twice)
    __shared__ float2 lds_ml[NW][RB];
    __shared__ int redo;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, lg = lane >> 4;
    const int w = div_by(blockIdx.x, p.by_hkv), hk = (int)blockIdx.x - w * p.HKV;
    Item it;
    if (!find_item<RB>(p, w, it) || it.chunk >= it.chunks) return;
    const int k0 = it.chunk * it.c, k1 = min(it.end - k0, it.c) + k0;   // the item's keys
    const int rows = min(it.n * p.G - it.rb * RB, RB);
    const int row = it.rb * RB + l16, qi = div_by(row, p.by_g);
    const int last = it.len - it.n + qi, last0 = it.len - it.n + div_by(it.rb * RB, p.by_g);   // this lane's row, and the block's first
    PageWalk<E4M3> walk;
    walk.row = p.c.table + (long)it.s * p.c.max_pages;
    const int start = k0 + 32 * wave;
    if (start < k1) walk.load(p, hk, start >> p.c.shift);
    bf16x8 qf[NKB] = {};
    if (l16 < rows) {
        const bf16_t* src = p.q + ((long)(it.tok + qi) * p.H + hk * p.G + row - qi * p.G) * DH;
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
    auto load = [&](Step& x, int kb) {
        walk.reach(p, hk, kb >> p.c.shift, (kb + 16) >> p.c.shift);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int key = kb + 16 * t, b = key >> p.c.shift;
            const int id = key < k1 ? walk.page(b) : -1;
            x.there[t] = id >= 0;
            if constexpr (E4M3) {   // (a page that holds none of the item's keys may have any scale)
                x.ks[t] = id >= 0 ? walk.kscale(b) : 1.f;
                x.vs[t] = id >= 0 ? walk.vscale(b) : 1.f;
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
        if (kb + 31 > last0 || kb + 32 > k1 || !x.there[0] || !x.there[1]) {   // some key is masked for some row
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
        floatx4 wt[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                wt[t][e] = __builtin_amdgcn_exp2f(st[t][e] - m);
                l += wt[t][e];
            }
            if constexpr (E4M3) wt[t] *= x.vs[t];
        }
        bf16x8 ph, pl;
        split_weights(wt[0], wt[1], ph, pl);
        int vb[8][CW / 2];   // bf16 pairs of channels
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < CW / 2; ++i) vb[j][i] = E4M3 ? fp8_pair(x.v[j][i / 2], i % 2) : x.v[j][E4M3 ? 0 : i];
#pragma unroll
        for (int n = 0; n < CW; ++n) {
            int4v va;
#pragma unroll
            for (int jj = 0; jj < 4; ++jj)
                va[jj] = __builtin_amdgcn_perm(vb[2 * jj + 1][n / 2], vb[2 * jj][n / 2], n % 2 ? 0x07060302 : 0x05040100);
            acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, va), ph, acc[n], 0, 0, 0);
            acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, va), pl, acc[n], 0, 0, 0);
        }
    };
    // DEPTH - 1 steps' loads are in flight while one is used
    constexpr int DEPTH = 256 / (DH * ESZ) + 1, NEXT = 32 * NW;
    Step ring[DEPTH];
    for (int kb = start - (DEPTH - 1) * NEXT; kb < k1; kb += NEXT * DEPTH) {
#pragma unroll
        for (int z = 0; z < DEPTH; ++z) {
            const int at = kb + NEXT * z, ahead = at + NEXT * (DEPTH - 1);
            if (ahead < k1) load(ring[(z + DEPTH - 1) % DEPTH], ahead);
            if (at >= start && at < k1) compute(ring[z], at);
        }
    }
    // the waves' sums: acc[n][e] is channel CW (4 lg + e) + n of query l16
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (l16 < rows) {
        if (lg == 0) lds_ml[wave][l16] = float2{m, l};
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int n = 0; n < CW; n += 4)
                *reinterpret_cast<floatx4*>(&lds_o[wave][l16][CW * (4 * lg + e) + n]) = floatx4{acc[n][e], acc[n + 1][e], acc[n + 2][e], acc[n + 3][e]};
    }
    if (k1 - 1 > last0) {
        // Some rows do not see some of the item's keys, but their weight of 0 does not hide a value that is not finite
        // (0 x NaN): where that left a sum that is not finite, the rows are done again without the matrix units.
        if (tid == 0) redo = 0;
        __syncthreads();
        float sum = 0.f;
#pragma unroll
        for (int n = 0; n < CW; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += 0.f * acc[n][e];
        if (l16 < rows && sum != 0.f) redo = 1;   // (0, or NaN)
        __syncthreads();
        if (redo) {
#pragma unroll 1
            for (int r = wave; r < rows; r += NW) {
                float o[8];
                plain_row<DH, CT>(p, it, hk, it.rb * RB + r, k0, k1, m, l, o);
                if (lane < NW) lds_ml[lane][r] = lane == 0 ? float2{m, l} : float2{LOWEST, 0.f};
                if (lane < DH / 8)
#pragma unroll
                    for (int z = 0; z < NW; ++z)
#pragma unroll
                        for (int e = 0; e < 8; ++e) lds_o[z][r][8 * lane + e] = z == 0 ? o[e] : 0.f;
            }
        }
    }
    __syncthreads();
    const int r = tid / 16, c0 = (tid % 16) * CW;
    if (r >= rows) return;
    float M = LOWEST, sum = 0.f;
    floatx4 o[CW / 4] = {};
#pragma unroll
    for (int z = 0; z < NW; ++z) M = fmaxf(M, lds_ml[z][r].x);
#pragma unroll
    for (int z = 0; z < NW; ++z) {
        const float a = __builtin_amdgcn_exp2f(lds_ml[z][r].x - M);
        sum += a * lds_ml[z][r].y;
#pragma unroll
        for (int n = 0; n < CW / 4; ++n) o[n] += a * f4(&lds_o[z][r][c0 + 4 * n]);
    }
    if (it.chunks == 1) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;   // no key: zeros
        const int rr = it.rb * RB + r, i = div_by(rr, p.by_g);
        bf16_t* dst = p.o + ((long)(it.tok + i) * p.H + hk * p.G + rr - i * p.G) * DH + c0;
#pragma unroll
        for (int n = 0; n < CW / 4; ++n) *reinterpret_cast<bf16x4*>(dst + 4 * n) = __builtin_convertvector(o[n] * inv, bf16x4);
    } else {
        const long slot = (long)blockIdx.x * RB + r;
        if (c0 == 0) p.pml[slot] = float2{M, sum};
#pragma unroll
        for (int n = 0; n < CW / 4; ++n) *reinterpret_cast<floatx4*>(p.po + slot * DH + c0 + 4 * n) = o[n];
    }
}

// ------------------------------------------------------------------ k_attn_tile: many rows
// Attention of blocks of 128 rows; bound by the matrix units and the softmax beside them.  Blocks of 64 keys and values
// lie in a double-buffered LDS ring (16-byte chunks XOR-swizzled as in k_attn_causal, whose products, running softmax and
// operand orders these are): a bf16 cache is copied there without registers, e4m3 codes are loaded a block ahead, made
// bf16 with their scale and stored.  A wave has two tiles of 16 rows, so that every K and V operand read from LDS feeds
// both tiles' products: LDS reads are what a block costs most beside the products (one tile a wave: 175 us against 164).
// Measured: 2048 new tokens behind 8192, 16 query heads of 128, 155 GFLOP in 166 us with joining, calls one after another (0.93
// PFLOP/s; a large product of a library reaches 1.2); in a trace of ten calls, at a lower clock, 177 us and 11 of joining.  From
// an e4m3 cache 195 us.  Products and the softmax's vector work of a SIMD's two waves hardly
// overlap; with the next block's scores formed beside this block's weights in one wave it took 181 us (all 256 registers),
// and 218 against 196 with the order prescribed to the compiler.
template <int DH, typename CT>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(2))) void k_attn_tile(PagedParams p) {
    constexpr bool E4M3 = sizeof(CT) == 1;
    constexpr int RB = AQ, QT = 2, NW = NT / 64, NCH = DH / 8, RPI = 64 / NCH, NKB = DH / 32, NDT = DH / 16, ESZ = sizeof(CT);
    // (a variable per ring slot: the compiler then sees that reads of one do not wait for the copies into the other)
    __shared__ __align__(16) bf16_t k_even[AKB * DH], v_even[AKB * DH], k_odd[AKB * DH], v_odd[AKB * DH];
    __shared__ int odd;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, lg = lane >> 4;
    const int w = div_by(blockIdx.x, p.by_hkv), hk = (int)blockIdx.x - w * p.HKV;
    Item it;
    if (!find_item<RB>(p, w, it) || it.chunk >= it.chunks) return;
    const int k0 = it.chunk * it.c, k1 = min(it.end - k0, it.c) + k0;
    const int rows = it.n * p.G, base = it.len - it.n;   // rows of the sequence; position of its first new token
    const int r0 = it.rb * RB + 16 * QT * wave;          // this wave's first row
    const int wlast = r0 < rows ? base + div_by(min(r0 + 16 * QT - 1, rows - 1), p.by_g) : -1;   // the last key that its rows see
    auto swz = [](int r) {
        return NCH == 16 ? (4 * (r & 3)) | (2 * ((r >> 2) & 1)) | ((r >> 3) & 1)
                         : (4 * ((r >> 1) & 1)) | (2 * ((r >> 2) & 1)) | ((r >> 3) & 1);
    };
    auto kq = [swz](int r, int cc) { return r * DH + (((cc >> 3) ^ swz(r)) << 3) + (cc & 7); };

    int last[QT], first[QT];   // the last keys of this lane's rows, and of a tile's first row
    bf16x8 qf[QT][NKB];
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        const int r = r0 + 16 * u + l16, qi = div_by(r, p.by_g);
        last[u] = base + qi;
        first[u] = base + div_by(r0 + 16 * u, p.by_g);
        const bf16_t* src = p.q + ((long)(it.tok + qi) * p.H + hk * p.G + r - qi * p.G) * DH;
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb) {
            qf[u][kb] = bf16x8{};
            if (r < rows) qf[u][kb] = *reinterpret_cast<const bf16x8*>(src + 32 * kb + 8 * lg);
        }
    }
    PageWalk<E4M3> walk;
    walk.row = p.c.table + (long)it.s * p.c.max_pages;
    if (k1 > k0) walk.load(p, hk, k0 >> p.c.shift);
    int there = 0, next_there = 0;   // bit t: keys 16 t .. of the block, and of the next one, are the item's and their page is there
    auto look = [&](int kb) {
        walk.reach(p, hk, kb >> p.c.shift, (kb + AKB - 1) >> p.c.shift);
        if (p.c.page >= AKB) {
            next_there = walk.page(kb >> p.c.shift) >= 0 ? 15 : 0;
        } else {
            next_there = 0;
#pragma unroll
            for (int t = 0; t < 4; ++t) next_there |= (kb + 16 * t < k1 && walk.page((kb + 16 * t) >> p.c.shift) >= 0) << t;
        }
    };
    // Rows of the block at key kb by descriptors whose offset 0 would be the block's first row: of the whole block where a page
    // holds it, else of the 16 rows around row r.  Rows past the item's keys, and of pages that are not there, read as zeros.
    auto describe = [&](int kb, int r, __amdgpu_buffer_rsrc_t& rk, __amdgpu_buffer_rsrc_t& rv, float& ks, float& vs) {
        const int g = p.c.page >= AKB ? 0 : r & ~15, span = p.c.page >= AKB ? AKB : 16, key = kb + g;
        const int id = key < k1 ? walk.page(key >> p.c.shift) : -1;
        if constexpr (E4M3) {   // (a page that holds none of the item's keys may have any scale)
            ks = id >= 0 ? walk.kscale(key >> p.c.shift) : 1.f;
            vs = id >= 0 ? walk.vscale(key >> p.c.shift) : 1.f;
        }
        const long at = (((((long)max(id, 0) * p.HKV + hk) << p.c.shift) + (key & (p.c.page - 1))) - g) * DH * ESZ;
        const uint32_t bytes = id >= 0 ? (uint32_t)(g + min(k1 - key, span)) * DH * ESZ : 0;
        rk = rsrc((const char*)p.c.k + at, bytes);
        rv = rsrc((const char*)p.c.v + at, bytes);
    };
    constexpr int NCW = AKB / RPI / NW;                   // bf16: this wave's 1 KB copies of K, and of V
    constexpr int PB = 16, NCB = AKB * DH / PB / NT;      // e4m3: bytes of a piece, and this thread's pieces of K, and of V
    static_assert(NCW >= 1 && NCB >= 1, "every thread copies the same share");
    int4v kc[E4M3 ? NCB : 1], vc[E4M3 ? NCB : 1];
    float kscale[E4M3 ? NCB : 1], vscale[E4M3 ? NCB : 1];   // of these pieces' page
    auto issue = [&](int kb, auto SLOT) {
        constexpr int sl = decltype(SLOT)::value;
        __amdgpu_buffer_rsrc_t rk, rv;
        float ks = 1.f, vs = 1.f;
        if constexpr (E4M3) {
#pragma unroll
            for (int c = 0; c < NCB; ++c) {
                const int row = 64 * (wave + NW * c) * PB / DH;   // the first of the wave's rows
                if (c == 0 || p.c.page < AKB) describe(kb, row, rk, rv, ks, vs);
                kscale[c] = ks;
                vscale[c] = vs;
                const int off = (tid + NT * c) * PB;
                kc[c] = __builtin_bit_cast(int4v, bload16(rk, off));
                vc[c] = __builtin_bit_cast(int4v, bload16(rv, off));
            }
        } else {
#pragma unroll
            for (int c = 0; c < NCW; ++c) {
                const int first = RPI * (wave + NW * c), r = first + lane / NCH;
                if (c == 0 || p.c.page < AKB) describe(kb, first, rk, rv, ks, vs);
                const int off = r * DH * 2 + (((lane % NCH) ^ swz(r)) << 4);
                bdma16(rk, &(sl ? k_odd : k_even)[first * DH], off);
                bdma16(rv, &(sl ? v_odd : v_even)[first * DH], off);
            }
        }
    };
    auto stage = [&](auto SLOT) {   // e4m3: the loaded codes into the ring
        constexpr int sl = decltype(SLOT)::value;
        if constexpr (E4M3) {
#pragma unroll
            for (int c = 0; c < NCB; ++c) {
                const int piece = tid + NT * c, r = piece * PB / DH, cc = piece * PB % DH;
#pragma unroll
                for (int z = 0; z < PB / 8; ++z) {
                    const int4v k4 = fp8_scaled(kc[c][2 * z], kc[c][2 * z + 1], kscale[c]), v4 = fp8_scaled(vc[c][2 * z], vc[c][2 * z + 1], vscale[c]);
                    *reinterpret_cast<int4v*>(&(sl ? k_odd : k_even)[kq(r, cc + 8 * z)]) = k4;
                    *reinterpret_cast<int4v*>(&(sl ? v_odd : v_even)[kq(r, cc + 8 * z)]) = v4;
                }
            }
        }
    };
    // The queries have to be there before the loop: a load still in flight at its head would make every block wait for the next
    // block's copies.
#pragma unroll
    for (int u = 0; u < QT; ++u)
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb) {
            int4v x = __builtin_bit_cast(int4v, qf[u][kb]);
            asm volatile("" : "+v"(x));
            qf[u][kb] = __builtin_bit_cast(bf16x8, x);
        }
    const float sl2 = p.scale_log2;
    float m[QT], l[QT];
    floatx4 oacc[QT][NDT];
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        m[u] = LOWEST;
        l[u] = 0.f;
#pragma unroll
        for (int t = 0; t < NDT; ++t) oacc[u][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    // A weight of 0 does not hide a value that is not finite (0 x NaN).  In the blocks from `part` on, where some rows do not
    // see a key that others see, such values are taken out, and added at the end, with their weight, to the rows that see them.
    const int all = base + div_by(it.rb * RB, p.by_g);   // the last key that every row sees
    const int part = all < k0 ? k0 : k0 + (all + 1 - k0) / AKB * AKB;
    if (tid == 0) odd = 0;
    auto block = [&](const int kb, auto SLOT) {
        constexpr int SL = decltype(SLOT)::value;
        if constexpr (!E4M3) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wave's copies of the block
        lds_barrier();   // everyone's; the other slot is no longer read
        there = next_there;
        if (kb + AKB < k1) {
            look(kb + AKB);
            issue(kb + AKB, Ic<1 - SL>{});
        }
        if (kb >= part) {
            bool found = false;
#pragma unroll
            for (int c = 0; c < AKB * DH / 8 / NT; ++c) {
                int4v* at = reinterpret_cast<int4v*>(&(SL ? v_odd : v_even)[(tid + NT * c) * 8]);
                int4v x = *at;
                bool any = false;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool hi = (x[i] & 0x7f800000) == 0x7f800000, lo = (x[i] & 0x7f80) == 0x7f80;
                    any = any || hi || lo;
                    x[i] = (hi ? 0 : x[i] & 0xffff0000) | (lo ? 0 : x[i] & 0xffff);
                }
                if (any) *at = x;
                found = found || any;
            }
            if (found) odd = 1;
            lds_barrier();
        }
        if (kb <= wlast) {
            const bf16_t* sk = SL ? k_odd : k_even;
            const bf16_t* sv = SL ? v_odd : v_even;
            floatx4 st[QT][4];   // S^T of query tile u: keys 16 t + 4 lg + e, query l16
#pragma unroll
            for (int u = 0; u < QT; ++u)
#pragma unroll
                for (int t = 0; t < 4; ++t) st[u][t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < NKB; ++i) {
                    const bf16x8 ka = *reinterpret_cast<const bf16x8*>(&sk[kq(16 * t + l16, 32 * i + 8 * lg)]);
#pragma unroll
                    for (int u = 0; u < QT; ++u) st[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qf[u][i], st[u][t], 0, 0, 0);
                }
            const bool whole = kb + AKB <= k1 && there == 15;
            float fs[QT], sum[QT];   // the weights are 2^(fs x - m); a lane's sum of them
            bf16x8 pf[QT][2];
            auto weigh = [&](int u) {
                sum[u] = 0.f;
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    floatx4 w[2];
#pragma unroll
                    for (int y = 0; y < 2; ++y)
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[y][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[u][2 * kk + y][e], fs[u], -m[u]));
                    pf[u][kk] = pack_bf16(w[0], w[1]);
                    sum[u] = sum_bf16(pf[u][kk], sum[u]);   // the rounded weights, which the products take
                }
            };
            bool up = false;
#pragma unroll
            for (int u = 0; u < QT; ++u) {
                fs[u] = sl2;
                if (!whole || kb + AKB - 1 > first[u]) {   // some key is masked for this tile
                    fs[u] = 1.f;
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int key = kb + 16 * t + 4 * lg + e;
                            st[u][t][e] = key > last[u] || key >= k1 || !((there >> t) & 1) ? -INFINITY : st[u][t][e] * sl2;
                        }
                }
                weigh(u);
                up = up || sum[u] > 4096.f;
            }
            // The reference m has to keep up with the scores only so far that the weights stay representable: it moves when
            // a lane's 16 weights sum to more than 2^12 (from a first m below every score: infinitely much), and only then is
            // a maximum taken, and the block's weights formed again.
            if (__builtin_amdgcn_ballot_w64(up)) {
#pragma unroll
                for (int u = 0; u < QT; ++u) {
                    float bm = m[u];
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) bm = fmaxf(bm, st[u][t][e] * fs[u]);
                    bm = fmaxf(bm, __shfl_xor(bm, 16, 64));
                    bm = fmaxf(bm, __shfl_xor(bm, 32, 64));
                    const float a = __builtin_amdgcn_exp2f(m[u] - bm);
#pragma unroll
                    for (int t = 0; t < NDT; ++t) oacc[u][t] *= a;
                    l[u] *= a;
                    m[u] = bm;
                    weigh(u);
                }
            }
#pragma unroll
            for (int u = 0; u < QT; ++u) l[u] += sum[u];
#pragma unroll
            for (int t = 0; t < NDT; ++t)
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    const int r = 32 * kk + 4 * lg + (l16 >> 2), c = 16 * t + 4 * (l16 & 3);
                    const bf16x8 va = join4(lds_tr8(&sv[kq(r, c)]), lds_tr8(&sv[kq(r + 16, c)]));
#pragma unroll
                    for (int u = 0; u < QT; ++u) oacc[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pf[u][kk], oacc[u][t], 0, 0, 0);
                }
        }
        if (kb + AKB < k1) stage(Ic<1 - SL>{});
    };
    if (k0 < k1) {
        look(k0);
        issue(k0, Ic<0>{});
        stage(Ic<0>{});
    }
    for (int kb = k0; kb < k1; kb += 2 * AKB) {
        block(kb, Ic<0>{});
        if (kb + AKB < k1) block(kb + AKB, Ic<1>{});
    }
    // (the barrier behind the last search of the values, if there was one, is ahead of this read)
#pragma unroll 1
    for (int key = part < k1 && odd ? part : k1; key < k1; ++key) {   // (rare)
        const int id = __builtin_amdgcn_readfirstlane(page_of(p.c, it.s, key >> p.c.shift));
        if (id < 0) continue;
        const long at = ((((long)id * p.HKV + hk) << p.c.shift) + (key & (p.c.page - 1))) * DH;
        float x[NDT][4];   // this lane's channels
        bool bad = false;
#pragma unroll
        for (int t = 0; t < NDT; ++t) {
            const CT* src = (const CT*)p.c.v + at + 16 * t + 4 * lg;
            short4v y;
            if constexpr (E4M3) {   // (as staged: a code's product with its scale may be what is not finite)
                const int4v z = fp8_scaled(*(const int*)src, 0, p.c.vs[(long)id * p.HKV + hk]);
                y = __builtin_bit_cast(short4v, (uint64_t)(uint32_t)z[0] | (uint64_t)(uint32_t)z[1] << 32);
            } else {
                y = *(const short4v*)src;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[t][e] = bf(y[e]);
                bad = bad || !(fabsf(x[t][e]) <= -LOWEST);
            }
        }
        if (!__builtin_amdgcn_ballot_w64(bad)) continue;
#pragma unroll
        for (int u = 0; u < QT; ++u) {
            float dot = 0.f;   // with this lane's share of the key
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb) {
                const CT* src = (const CT*)p.c.k + at + 32 * kb + 8 * lg;
                float k[8];
                if constexpr (E4M3) {
                    from_e4m3(*(const uint64_t*)src, k);
                } else {
                    Chunk8<bf16_t> y;
                    y.load(src);
                    y.get(k);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) dot += (float)qf[u][kb][e] * k[e];
            }
            if constexpr (E4M3) dot *= p.c.ks[(long)id * p.HKV + hk];
            dot += __shfl_xor(dot, 16, 64);
            dot += __shfl_xor(dot, 32, 64);
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(dot, sl2, -m[u]));
#pragma unroll
            for (int t = 0; t < NDT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (key <= last[u] && !(fabsf(x[t][e]) <= -LOWEST)) oacc[u][t][e] += w * x[t][e];
        }
    }
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        l[u] += __shfl_xor(l[u], 16, 64);
        l[u] += __shfl_xor(l[u], 32, 64);
        const int r = r0 + 16 * u + l16;
        if (r >= rows) continue;
        if (it.chunks == 1) {
            const float inv = l[u] == 0.f ? 0.f : 1.f / l[u];   // no key: zeros
            const int i = div_by(r, p.by_g);
            bf16_t* dst = p.o + ((long)(it.tok + i) * p.H + hk * p.G + r - i * p.G) * DH + 4 * lg;
#pragma unroll
            for (int t = 0; t < NDT; ++t) *reinterpret_cast<bf16x4*>(dst + 16 * t) = __builtin_convertvector(oacc[u][t] * inv, bf16x4);
        } else {
            const long slot = (long)blockIdx.x * RB + (r - it.rb * RB);
            if (lg == 0) p.pml[slot] = float2{m[u], l[u]};
#pragma unroll
            for (int t = 0; t < NDT; ++t) *reinterpret_cast<floatx4*>(p.po + slot * DH + 16 * t + 4 * lg) = oacc[u][t];
        }
    }
}

// ------------------------------------------------------------------ k_attn_join
// The sum of a row's chunks' partial sums, over loads of 4 channels a lane, lanes and waves in a fixed order (so that the
// result does not depend on which chunk ended first).  (The last workgroup of a block adding up at its end, found by flags
// stored past the caches, was slower: 64 sequences e4m3 81 us against 78, 16 sequences' 4 tokens 38 against 23.)
// Blocks of 16 rows may have many chunks: a workgroup a row (blockIdx.y), its waves sharing them.  Bound by latency: the
// launch, the search for the item and one round trip to memory; 5.6 us for 63 chunks.
template <int DH>
__global__ __launch_bounds__(NT) void k_attn_join(PagedParams p) {
    constexpr int RB = 16, LPR = DH / 4, SUB = 64 / LPR, NW = NT / 64;   // lanes per row; chunks that a wave's load takes at once
    __shared__ __align__(16) float red[NW][DH];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int w = div_by(blockIdx.x, p.by_hkv), hk = (int)blockIdx.x - w * p.HKV, c4 = 4 * (lane % LPR), r = blockIdx.y;
    Item it;
    if (!find_item<RB, true>(p, w, it) || it.chunks == 1) return;
    const int rr = it.rb * RB + r, chunks = it.chunks;
    if (rr >= it.n * p.G) return;
    auto slot = [&](int j) { return ((long)item_of(it, j) * p.HKV + hk) * RB + r; };
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
            if (j < chunks) y[k] = f4(p.po + slot(j) * DH + c4);
        }
        float2 ml = {LOWEST, 0.f};   // of chunk j0 + lane
        if (j0 + lane < chunks) ml = p.pml[slot(j0 + lane)];
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
    const int i = div_by(rr, p.by_g);
    bf16_t* dst = p.o + ((long)(it.tok + i) * p.H + hk * p.G + rr - i * p.G) * DH + c4;
    *reinterpret_cast<bf16x4*>(dst) = __builtin_convertvector(o * inv, bf16x4);
}

// Blocks of 128 rows have few chunks, mostly two: DH / 4 lanes a row, 16 rows (blockIdx.y) a workgroup.
template <int DH>
__global__ __launch_bounds__(NT) void k_attn_join_tile(PagedParams p) {
    constexpr int RB = AQ, LPR = DH / 4, NG = NT / LPR, ROWS = 16, PASS = ROWS / NG;
    const int g = blockIdx.y * ROWS + threadIdx.x / LPR, c4 = 4 * (threadIdx.x % LPR);
    const int w = div_by(blockIdx.x, p.by_hkv), hk = (int)blockIdx.x - w * p.HKV;
    Item it;
    if (!find_item<RB, true>(p, w, it) || it.chunks == 1) return;
    const int rows = min(it.n * p.G - it.rb * RB, RB), chunks = it.chunks;
    auto slot = [&](int j, int r) { return ((long)item_of(it, j) * p.HKV + hk) * RB + r; };
    float M[PASS], sum[PASS];
    floatx4 o[PASS];
#pragma unroll
    for (int i = 0; i < PASS; ++i) {
        M[i] = LOWEST;
        sum[i] = 0.f;
        o[i] = floatx4{0.f, 0.f, 0.f, 0.f};
        const int r = g + i * NG;
        for (int j = threadIdx.x % LPR; j < chunks && r < rows; j += LPR) M[i] = fmaxf(M[i], p.pml[slot(j, r)].x);
#pragma unroll
        for (int off = 1; off < LPR; off <<= 1) M[i] = fmaxf(M[i], __shfl_xor(M[i], off, 64));
    }
#pragma unroll 8
    for (int j = 0; j < chunks; ++j)
#pragma unroll
        for (int i = 0; i < PASS; ++i) {
            const int r = min(g + i * NG, rows - 1);   // (rows past the block's are not written)
            const float2 ml = p.pml[slot(j, r)];
            const floatx4 y = f4(p.po + slot(j, r) * DH + c4);
            const float w = __builtin_amdgcn_exp2f(ml.x - M[i]);
            sum[i] += w * ml.y;
            o[i] += w * y;
        }
#pragma unroll
    for (int i = 0; i < PASS; ++i) {
        const int r = g + i * NG, rr = it.rb * RB + r;
        if (r >= rows) break;
        const float inv = sum[i] == 0.f ? 0.f : 1.f / sum[i];
        const int qi = div_by(rr, p.by_g);
        bf16_t* dst = p.o + ((long)(it.tok + qi) * p.H + hk * p.G + rr - qi * p.G) * DH + c4;
        *reinterpret_cast<bf16x4*>(dst) = __builtin_convertvector(o[i] * inv, bf16x4);
    }
}
