// cf_logprobs.hip -- log probabilities of given tokens (classes), entropy and
// the most probable alternatives from rows of logits z, and the gradient.
//
//   m = max_j z_j,  s = sum_j exp(z_j - m),  log p_j = (z_j - m) - log s
//   H = -sum_j p_j log p_j = log s - 1/s sum_j exp(z_j - m) (z_j - m)
//   dz_j = g (1[j = token] - p_j) - h p_j (log p_j + H)     for gradients g of log p, h of H
//
// The forward pass reads the logits once: every thread keeps the running
// maximum of its share of the row with the two sums relative to it (fp32;
// exponentials in base 2) and rescales them when the maximum grows; the
// threads' triples are joined at the end.  Few rows are cut into chunks for
// workgroups of their own, whose triples a second launch joins.
//
// A logit of -inf has probability 0 and adds nothing.  A row with nothing else
// has log p = -inf, H = 0 and no gradient; one with +inf or NaN has NaN
// everywhere.  References to the maximum stay at or above the lowest finite
// number, so that rows masked with it are as good as any other.
//
// Rows of up to 4096 logits (2048 in fp32) stay in the registers of a wave or
// of 8, 16 or 32 of its lanes (65536 rows of 100 with five alternatives: 14 us,
// 50 with a wave each, 360 with a workgroup).
//
// Alternatives of longer rows: the n-th largest of the 64 maxima over four
// threads each bounds the n-th largest logit from below, so only the few threads
// whose maximum reaches it look at their share again and collect what does.
// Equal logits rank by index; where more are equal than fit the list (a row with
// few classes left), those above the bound are collected and the equal ones taken
// in the order of the row.
//
// Measured on MI355X, where a copy of 2 GiB moves 4.9 TB/s: 4096 rows of 100003 in
// bf16 forward 150 us among calls of its kind (5.5 TB/s; VALU 83% busy), 177 to 188
// behind a backward pass, which takes 271 to 278 (6 TB/s); one row of 131072 with
// eight alternatives 5.6 us in 64 workgroups and 4.0 us to join them; 128 rows of
// 1000 with five 6.1 us.  The last two are chains: load, maximum, join,
// alternatives, the logit asked for.  Rows of a wave each are bound by instructions
// where they have alternatives, of which a key for every logit is the most: 60000
// rows of 1000 with five or eight 65 us (none: 33), 10000 of 4000 with eight 41
// (18), 20000 of 2000 with twenty 40 (19), 65536 of 100 with five 14 (7.6).
#include "cf_rows.h"
#include "cf_kernels.h"
#include "cf_train.h"

namespace cf {

namespace {

constexpr float LOG2E = 1.44269504f, LN2 = 0.693147181f, LOWEST = -3.40282347e38f;
// exponents below this give 0; also stands in for -inf, whose product with 0 is not 0
constexpr float FLOOR2 = -1000.0f;

// 16 bytes of logits: VE values, of which n are before `end` (the rest -inf).
// `end` is the row's end or, in a chunk, a multiple of 8.
template <typename T>
struct Z16 {
    typedef uint16_t elem;
    static constexpr int VE = 8;
    typedef u32x4 raw;
    static __device__ __forceinline__ raw load(const elem *row, int i, int end) { return load8(row, i, end); }
    static __device__ __forceinline__ void values(const raw &r, int n, float *z) {
        unpack8<T>(r, z);
        if (n < 8)
#pragma unroll
            for (int i = 0; i < 8; i++)
                z[i] = i < n ? z[i] : -INFINITY;
    }
    static __device__ __forceinline__ float one(const elem *p) { return T::lo(*p); }
    static __device__ __forceinline__ void store(elem *row, int i, int end, const float *z) {
        store8(row, i, end, pack8<T>(z));
    }
};
struct Z32 {
    typedef float elem;
    static constexpr int VE = 4;
    typedef float4v raw;
    struct __attribute__((packed, aligned(4))) Any {
        float4v v;
    };
    static __device__ __forceinline__ raw load(const elem *row, int at, int end) {
        const elem *const p = row + at;
        const int n = end - at;
        if (n >= 4)
            return reinterpret_cast<const Any *>(p)->v;
        raw r = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 3; i++)
            if (i < n)
                r[i] = p[i];
        return r;
    }
    static __device__ __forceinline__ void values(const raw &r, int n, float *z) {
#pragma unroll
        for (int i = 0; i < 4; i++)
            z[i] = i < n ? r[i] : -INFINITY;
    }
    static __device__ __forceinline__ float one(const elem *p) { return *p; }
    static __device__ __forceinline__ void store(elem *row, int at, int end, const float *z) {
        elem *const p = row + at;
        const int n = end - at;
        if (n >= 4) {
            reinterpret_cast<Any *>(p)->v = float4v{z[0], z[1], z[2], z[3]};
            return;
        }
#pragma unroll
        for (int i = 0; i < 3; i++)
            if (i < n)
                p[i] = z[i];
    }
};

// ---------------------------------------------------------------------------
// Maximum m (NaN if any logit is), s and t = sum exp2(d) d of the logits seen,
// d = (z - max(m, LOWEST)) log2 e.
struct Stat {
    float m, s, t;
};
__device__ __forceinline__ float ref_of(float m) { return fmaxf(m, LOWEST); }

// the sums of a relative to a maximum m >= a.m instead
__device__ __forceinline__ void rebase(Stat &a, float m) {
    const float d = fmaxf((ref_of(a.m) - ref_of(m)) * LOG2E, FLOOR2), f = __builtin_amdgcn_exp2f(d);
    a.t = f * fmaf(d, a.s, a.t);
    a.s *= f;
    a.m = m;
}

template <int N>
__device__ __forceinline__ void add(Stat &a, const float *z) {
    float m = a.m;
#pragma unroll
    for (int i = 0; i < N; i++)
        m = Max::of(m, z[i]);
    if (!(m == a.m))
        rebase(a, m);
    const float ref = ref_of(m);
#pragma unroll
    for (int i = 0; i < N; i++) {
        const float d = fmaxf((z[i] - ref) * LOG2E, FLOOR2), e = __builtin_amdgcn_exp2f(d);
        a.s += e;
        a.t = fmaf(e, d, a.t);
    }
}

// of G neighbouring lanes
template <int G = 64>
__device__ __forceinline__ Stat wave_join(Stat a) {
    const float m = lanes<Max, G>(a.m);
    rebase(a, m);
    return {m, lanes<Add, G>(a.s), lanes<Add, G>(a.t)};
}

// ---------------------------------------------------------------------------
// Order of the alternatives: larger logits first, NaN before all, equal ones
// by index.  Key 0 is none.
__device__ __forceinline__ uint64_t key_of(float z, uint32_t i) {
    const uint32_t u = __builtin_bit_cast(uint32_t, z + 0.0f);  // -0 equals 0
    const uint32_t o = z != z ? 0xffffffffu : u & 0x80000000u ? ~u : u | 0x80000000u;
    return (uint64_t)o << 32 | (0xffffffffu - i);
}
__device__ __forceinline__ float logit_of(uint64_t k) {
    const uint32_t o = (uint32_t)(k >> 32);
    return o == 0xffffffffu ? NAN : __builtin_bit_cast(float, o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int64_t index_of(uint64_t k) { return (int64_t)(0xffffffffu - (uint32_t)k); }

template <int CTRL>
__device__ __forceinline__ uint64_t dpp64(uint64_t k) {
    const int lo = (int)(uint32_t)k, hi = (int)(uint32_t)(k >> 32);
    return (uint64_t)(uint32_t)__builtin_amdgcn_update_dpp(hi, hi, CTRL, 0xf, 0xf, true) << 32 |
           (uint32_t)__builtin_amdgcn_update_dpp(lo, lo, CTRL, 0xf, 0xf, true);
}
__device__ __forceinline__ uint64_t later(uint64_t a, uint64_t b) { return a > b ? a : b; }
template <int G = 64>
__device__ __forceinline__ uint64_t wave_max(uint64_t k) {
    k = later(k, dpp64<DPP_XOR1>(k));
    k = later(k, dpp64<DPP_XOR2>(k));
    k = later(k, dpp64<DPP_MIRROR8>(k));
    if constexpr (G >= 16)
        k = later(k, dpp64<DPP_MIRROR16>(k));
    if constexpr (G >= 32) {
        const auto l = __builtin_amdgcn_permlane16_swap((uint32_t)k, (uint32_t)k, false, false);
        const auto h = __builtin_amdgcn_permlane16_swap((uint32_t)(k >> 32), (uint32_t)(k >> 32), false, false);
        k = later((uint64_t)h[0] << 32 | (uint32_t)l[0], (uint64_t)h[1] << 32 | (uint32_t)l[1]);
    }
    if constexpr (G >= 64) {
        const auto l = __builtin_amdgcn_permlane32_swap((uint32_t)k, (uint32_t)k, false, false);
        const auto h = __builtin_amdgcn_permlane32_swap((uint32_t)(k >> 32), (uint32_t)(k >> 32), false, false);
        k = later((uint64_t)h[0] << 32 | (uint32_t)l[0], (uint64_t)h[1] << 32 | (uint32_t)l[1]);
    }
    return k;
}

struct Args {
    const void *z;
    const int64_t *tokens;
    float *logp, *entropy;
    float2 *stats;
    float *top_logp;
    int64_t *top_ids;
    float4 *part;        // [rows][chunks]: m, s, t
    uint64_t *part_key;  // [rows][chunks][top], in order
    int64_t ldz;
    int V, top, chunks, chunk;  // logits of a chunk, a multiple of 8
};

// The token that a row asks about and its logit, loaded ahead by the thread that
// finishes the row.
struct Asked {
    int64_t token;
    float z;
};
template <typename Z>
__device__ __forceinline__ Asked ask(const Args &a, int64_t row) {
    Asked q = {a.tokens ? a.tokens[row] : -1, 0.0f};
    if (q.token >= 0 && q.token < a.V)
        q.z = Z::one((const typename Z::elem *)a.z + row * a.ldz + q.token);
    return q;
}

// what a row's sums say; one thread
__device__ __forceinline__ void finish(const Args &a, int64_t row, const Stat &s, const Asked &q) {
    const bool bad = !(s.m < INFINITY), empty = s.s == 0.0f;
    const float ls = bad ? NAN : empty ? 0.0f : logf(s.s);
    if (a.logp)
        a.logp[row] = q.token >= a.V ? NAN : q.token < 0 ? 0.0f : bad ? NAN : (q.z - ref_of(s.m)) - ls;
    a.entropy[row] = bad ? NAN : empty ? 0.0f : fmaxf(ls - LN2 * (s.t / s.s), 0.0f);
    if (a.stats)
        a.stats[row] = bad ? make_float2(NAN, NAN) : empty ? make_float2(-INFINITY, 0.0f) : make_float2(s.m, ls);
}

// one alternative of a row
__device__ __forceinline__ void put_top(const Args &a, int64_t row, int n, uint64_t key, const Stat &s) {
    const bool bad = !(s.m < INFINITY);
    const float z = logit_of(key);
    a.top_logp[row * a.top + n] = bad ? NAN : s.s == 0.0f ? z : (z - ref_of(s.m)) - logf(s.s);
    a.top_ids[row * a.top + n] = index_of(key);
}

constexpr int TH = 256;    // threads of a workgroup
constexpr int LIST = 512;  // logits collected before equal ones are counted

// The logits [begin, end) of a row in vectors that start at multiples of 16
// bytes, whatever the row's own start: the first vector holds what comes
// before the first such place (4096 rows of 100003 in bf16: 170 -> 150 us).
// Vector v has n logits from index i on (none: n <= 0).
template <typename Z>
struct Piece {
    const typename Z::elem *z;
    int begin, end, V, pad;
    __device__ __forceinline__ Piece(const typename Z::elem *row, int b, int e, int len)
        : z(row), begin(b), end(e), V(len), pad((int)((uintptr_t)(row + b) & 15u) / (int)sizeof(*row)) {}
    struct At {
        int i, n;
    };
    __device__ __forceinline__ At at(int v) const {
        const int i = begin - pad + v * Z::VE;
        const int from = i > begin ? i : begin, to = i + Z::VE < end ? i + Z::VE : end;
        return {from, to - from};
    }
    __device__ __forceinline__ int vectors() const { return (end - begin + pad + Z::VE - 1) / Z::VE; }
    // the logits' bits, and the logits (-inf past n)
    __device__ __forceinline__ typename Z::raw load(const At &a) const { return Z::load(z, a.i, V); }
    __device__ __forceinline__ void values(const At &a, float *x) const { Z::values(load(a), a.n, x); }
};

// f(value, index) for every logit of this thread's share.
template <typename Z, typename F>
__device__ __forceinline__ void each(const Piece<Z> &p, F &&f) {
    for (int v = threadIdx.x; v < p.vectors(); v += TH) {
        const auto a = p.at(v);
        float x[Z::VE];
        p.values(a, x);
#pragma unroll
        for (int e = 0; e < Z::VE; e++)
            if (e < a.n)
                f(x[e], (uint32_t)(a.i + e));
    }
}

struct TopSpace {
    alignas(16) float gm[64];  // read by fours
    uint64_t list[LIST];
    uint64_t out[TOP_MAX];
    uint64_t best[TH / 64];
    int n, threads, cnt[TH / 64];
    uint8_t who[TH];
};
static_assert(alignof(TopSpace) % alignof(float4) == 0 && offsetof(TopSpace, gm) % alignof(float4) == 0,
              "gm is read as float4");

// Logits of the piece that `wanted` takes, from the shares of the threads
// that say `mine`, into sp.list; their number in sp.n (which may pass LIST).
// The whole workgroup reads those shares, a vector a thread, so that a row's
// length does not become a chain of loads.
template <typename Z, typename F>
__device__ void collect(const Piece<Z> &p, bool mine, TopSpace &sp, F &&wanted) {
    const int tid = threadIdx.x;
    if (tid == 0)
        sp.n = sp.threads = 0;
    __syncthreads();
    if (mine)
        sp.who[atomicAdd(&sp.threads, 1)] = (uint8_t)tid;
    __syncthreads();
    const unsigned each = (unsigned)(p.vectors() + TH - 1) / TH, all = sp.threads * each;
    for (unsigned w = tid; w < all; w += TH) {
        // enough to know that they are too many: a row of equal logits would add
        // every one (512 rows of 50257, one of them masked whole: 49 us, so 19)
        if (*(volatile int *)&sp.n > LIST)
            break;
        const unsigned t = w / each;
        const int v = (int)((w - t * each) * TH + sp.who[t]);
        if (v >= p.vectors())
            continue;
        const auto a = p.at(v);
        float x[Z::VE];
        p.values(a, x);
#pragma unroll
        for (int e = 0; e < Z::VE; e++)
            if (e < a.n && wanted(x[e])) {
                const int at = atomicAdd(&sp.n, 1);
                if (at < LIST)
                    sp.list[at] = key_of(x[e], (uint32_t)(a.i + e));
            }
    }
    __syncthreads();
}

// The `top` first logits of the piece in order into sp.out (0 where there
// are fewer); tm is the maximum of this thread's share and x its last vector.
// Every thread calls it and may read sp.out afterwards.
template <typename Z>
__device__ void find_top(const Piece<Z> &p, int top, float tm, const float *x, TopSpace &sp) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const float g = lanes<Max, 4>(tm);
    if ((tid & 3) == 0)
        sp.gm[tid >> 2] = g;
    if (tid == 0)
        sp.n = 0;
    if (tid < top)
        sp.out[tid] = 0;
    __syncthreads();
    // the n-th largest of the 64 maxima: the least one with fewer than n above it
    const float mine = sp.gm[lane];
    int above = 0;
    bool nan = false;
#pragma unroll
    for (int j = 0; j < 64; j += 4) {
        const float4 o = *reinterpret_cast<const float4 *>(&sp.gm[j]);
        above += (o.x > mine) + (o.y > mine) + (o.z > mine) + (o.w > mine);
        nan |= o.x != o.x || o.y != o.y || o.z != o.z || o.w != o.w;
    }
    const float bound = -lanes<Max, 64>(above < top ? -mine : -INFINITY);
    // nan is the same in every thread
    bool done = false;
    if (!nan) {
        if (p.vectors() <= TH) {  // the shares are at hand (one row of 131072 9.7 us a call, read again 9.9)
            const auto a = p.at(tid);
            if (tm >= bound)
#pragma unroll
                for (int e = 0; e < Z::VE; e++)
                    if (e < a.n && x[e] >= bound) {
                        const int at = atomicAdd(&sp.n, 1);
                        if (at < LIST)
                            sp.list[at] = key_of(x[e], (uint32_t)(a.i + e));
                    }
            __syncthreads();
        } else {
            collect<Z>(p, tm >= bound, sp, [&](float v) { return v >= bound; });
        }
        int n = sp.n;
        done = n <= LIST;
        if (!done) {  // many are equal: those above the bound, then the first of the equal ones
            __syncthreads();
            collect<Z>(p, tm > bound, sp, [&](float v) { return v > bound; });
            n = sp.n;
            done = n + TOP_MAX <= LIST;
            if (done && n < top) {
                const int above_n = n, want = top - n;
                int found = 0;
                for (int v0 = 0; v0 < p.vectors() && found < want; v0 += TH) {
                    typename Piece<Z>::At a = {0, 0};
                    unsigned eq = 0;
                    if (v0 + tid < p.vectors()) {
                        a = p.at(v0 + tid);
                        float x[Z::VE];
                        p.values(a, x);
#pragma unroll
                        for (int e = 0; e < Z::VE; e++)
                            eq |= (unsigned)(x[e] == bound && e < a.n) << e;
                    }
                    int c = __popc(eq), before = c;
#pragma unroll
                    for (int o = 1; o < 64; o <<= 1) {
                        const int up = __shfl_up(before, o);
                        before += lane >= o ? up : 0;
                    }
                    if (lane == 63)
                        sp.cnt[wave] = before;
                    __syncthreads();
                    int at = found + before - c, all = 0;
#pragma unroll
                    for (int w = 0; w < TH / 64; w++) {
                        at += w < wave ? sp.cnt[w] : 0;
                        all += sp.cnt[w];
                    }
#pragma unroll
                    for (int e = 0; e < Z::VE; e++)
                        if (eq >> e & 1) {
                            if (at < want)
                                sp.list[above_n + at] = key_of(bound, (uint32_t)(a.i + e));
                            at++;
                        }
                    found += all;
                    __syncthreads();
                }
                n += found < want ? found : want;
            }
        }
        if (done) {
            for (int i = tid; i < n; i += TH) {
                const uint64_t k = sp.list[i];
                int rank = 0;
                for (int j = 0; j < n; j++)
                    rank += sp.list[j] > k;
                if (rank < top)
                    sp.out[rank] = k;
            }
        }
    }
    if (!done) {  // NaN, or hundreds above the bound in few threads: one pass for each
        uint64_t last = ~0ull;
        bool first = true;
        for (int r = 0; r < top; r++) {
            uint64_t best = 0;
            each<Z>(p, [&](float v, uint32_t i) {
                const uint64_t k = key_of(v, i);
                best = (first || k < last) && k > best ? k : best;
            });
            best = wave_max(best);
            __syncthreads();
            if (lane == 0)
                sp.best[wave] = best;
            __syncthreads();
            best = sp.best[0];
#pragma unroll
            for (int w = 1; w < TH / 64; w++)
                best = later(best, sp.best[w]);
            if (tid == 0)
                sp.out[r] = best;
            if (best == 0)
                break;
            last = best;
            first = false;
        }
    }
    __syncthreads();
}

// One chunk of one row a workgroup, NV vectors a thread loaded together; a row
// of one chunk is finished here.
template <typename Z, bool TOP, int NV>
__global__ __launch_bounds__(TH) void log_probs_kernel(Args a) {
    __shared__ Stat join[TH / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = blockIdx.x / (unsigned)a.chunks;
    const int part = (int)(blockIdx.x - (unsigned)row * (unsigned)a.chunks);
    const typename Z::elem *const z = (const typename Z::elem *)a.z + row * a.ldz;
    const int begin = part * a.chunk, end = a.V - begin < a.chunk ? a.V : begin + a.chunk;
    const Piece<Z> piece(z, begin, end, a.V);
    const int vectors = piece.vectors();

    Stat st = {-INFINITY, 0.0f, 0.0f};
    Asked asked = {-1, 0.0f};
    if (tid == 0 && a.chunks == 1)
        asked = ask<Z>(a, row);
    typename Z::raw next[NV] = {};
    auto fetch = [&](int v) {
#pragma unroll
        for (int u = 0; u < NV; u++)
            if (v + u * TH < vectors)
                next[u] = piece.load(piece.at(v + u * TH));
    };
    int v = tid;
    fetch(v);
    float x[NV * Z::VE];
    for (; v < vectors; v += NV * TH) {
        typename Z::raw cur[NV];
#pragma unroll
        for (int u = 0; u < NV; u++)
            cur[u] = next[u];
        fetch(v + NV * TH);
#pragma unroll
        for (int u = 0; u < NV; u++)
            Z::values(cur[u], piece.at(v + u * TH).n, x + u * Z::VE);
        add<NV * Z::VE>(st, x);
    }
    const float tm = st.m;
    st = wave_join(st);
    if (lane == 0)
        join[wave] = st;
    __syncthreads();
    float m = join[0].m;
#pragma unroll
    for (int w = 1; w < TH / 64; w++)
        m = Max::of(m, join[w].m);
    Stat all = {m, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < TH / 64; w++) {
        Stat o = join[w];
        rebase(o, m);
        all.s += o.s;
        all.t += o.t;
    }
    if constexpr (TOP) {
        __shared__ TopSpace sp;
        find_top<Z>(piece, a.top, tm, x, sp);
        if (tid < a.top) {
            if (a.chunks > 1)
                a.part_key[(row * a.chunks + part) * a.top + tid] = sp.out[tid];
            else
                put_top(a, row, tid, sp.out[tid], all);
        }
    }
    if (tid == 0) {
        if (a.chunks > 1)
            a.part[row * a.chunks + part] = make_float4(all.m, all.s, all.t, 0.0f);
        else
            finish(a, row, all, asked);
    }
}

// ---------------------------------------------------------------------------
// Short rows: G lanes of a wave take one whole, NV vectors a lane, all in
// registers and without a barrier.  Few alternatives are found one after the
// other: the largest key of the group, then the next of the lane that held it.
//
// Keys of 16-bit logits fit 32 bits: the low 13 bits of their fp32 form are
// zeros and take the index (V below 8192).
template <typename Z>
struct WaveKey {
    typedef uint64_t key;
    static constexpr int FEW = 3;
    static __device__ __forceinline__ key of(float z, int i, bool) { return key_of(z, (uint32_t)i); }
    template <int G>
    static __device__ __forceinline__ key best(key k) {
        return wave_max<G>(k);
    }
    static __device__ __forceinline__ uint64_t wide(key k) { return k; }
};
template <typename T>
struct WaveKey<Z16<T>> {
    typedef uint32_t key;
    static constexpr int FEW = 5;
    static constexpr uint32_t INDEX = 0x1fffu;
    static __device__ __forceinline__ key of(float z, int i, bool nan) {
        const uint32_t u = __builtin_bit_cast(uint32_t, z + 0.0f);  // -0 equals 0
        uint32_t o = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
        if (nan)  // of the row: of any sign, before all
            o = z != z ? 0xffffffffu : o;
        return (o & ~INDEX) | (INDEX - (uint32_t)i);
    }
    template <int CTRL>
    static __device__ __forceinline__ key step(key k) {
        const key o = (key)__builtin_amdgcn_update_dpp((int)k, (int)k, CTRL, 0xf, 0xf, true);
        return k > o ? k : o;
    }
    template <int G>
    static __device__ __forceinline__ key best(key k) {
        k = step<DPP_MIRROR8>(step<DPP_XOR2>(step<DPP_XOR1>(k)));
        if constexpr (G >= 16)
            k = step<DPP_MIRROR16>(k);
        if constexpr (G >= 32) {
            const auto a = __builtin_amdgcn_permlane16_swap(k, k, false, false);
            k = a[0] > a[1] ? a[0] : a[1];
        }
        if constexpr (G >= 64) {
            const auto b = __builtin_amdgcn_permlane32_swap(k, k, false, false);
            k = b[0] > b[1] ? b[0] : b[1];
        }
        return k;
    }
    static __device__ __forceinline__ uint64_t wide(key k) {
        const uint32_t o = k & ~INDEX;
        // the value's low bits, which the index took: zeros of a positive
        // number, ones (it is stored inverted) of a negative one
        const uint32_t whole = o == ~INDEX ? 0xffffffffu : o & 0x80000000u ? o : o | INDEX;
        return (uint64_t)whole << 32 | (0xffffffffu - (INDEX - (k & INDEX)));
    }
};

// Orders a wave's LDS writes and the reads of other lanes' after them.
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A few alternatives of a wave's row (K::FEW) are found one after the other, more
// among the logits that reach the n-th largest of the lanes' maxima, collected and
// ranked by counting.  60000 rows of 1000, one after the other and collected: bf16
// four 60 and 65 us, five 65 and 66, six 69 and 66, eight 78 and 66; fp32, whose
// keys are twice as wide, three 75 and 79, four 85 and 79, eight 124 and 80.  10000 of
// 4000 in bf16: five 40 and 41, six 43 and 41; 10000 of 400 in fp32: three 11.4 and
// 12.6, five 13.9 and 12.8.  Up to 256 are collected, as many as reach the bound in
// a row of equal logits; up to 64 of short rows in 16 bits, where the way for few
// takes less than ranking more (128 rows of 400, one of them masked whole, twenty:
// 7.3 us against 10.7).
template <typename Z, int G, int NV, bool TOP>
__global__ __launch_bounds__(256) void log_probs_wave_kernel(Args a, int64_t rows) {
    typedef WaveKey<Z> K;
    const int lane = threadIdx.x % G;  // of the group
    const int group = G == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / G) : threadIdx.x / G;
    const int64_t row = (int64_t)blockIdx.x * (256 / G) + group;
    if (row >= rows)  // whole groups: no exchange crosses them
        return;
    const typename Z::elem *const z = (const typename Z::elem *)a.z + row * a.ldz;
    float x[NV * Z::VE];
    typename Z::raw raw[NV];
#pragma unroll
    for (int v = 0; v < NV; v++)
        raw[v] = Z::load(z, (v * G + lane) * Z::VE, a.V);
    const Asked asked = ask<Z>(a, row);
#pragma unroll
    for (int v = 0; v < NV; v++)
        Z::values(raw[v], a.V - (v * G + lane) * Z::VE, x + v * Z::VE);
    Stat st = {-INFINITY, 0.0f, 0.0f};
    add<NV * Z::VE>(st, x);
    st = wave_join<G>(st);
    if constexpr (TOP) {
        const bool nan = st.m != st.m;  // the same in all lanes of the group
        typename K::key k[NV * Z::VE], mine = 0, top = 0;
#pragma unroll
        for (int i = 0; i < NV * Z::VE; i++) {
            const int at = (i / Z::VE * G + lane) * Z::VE + i % Z::VE;
            k[i] = at < a.V ? K::of(x[i], at, nan) : 0;
            top = k[i] > top ? k[i] : top;
        }
        int from = 0;
        if constexpr (G == 64)
            if (a.top > K::FEW) {
                typedef typename K::key Key;
                constexpr int WAVE_LIST = Z::VE == 8 && NV <= 2 ? 64 : 256;
                __shared__ __align__(16) Key heads[4][64], list[4][WAVE_LIST];
                Key *const head = heads[group], *const found = list[group];
                head[lane] = top;
                wave_fence();
                int above = 0;
#pragma unroll 16
                for (int j = 0; j < 64; j++)
                    above += head[j] > top;
                // the least of the n largest maxima (keys differ but for 0)
                const Key bound = ~K::template best<64>(above < a.top ? (Key)~top : (Key)0);
                int count = 0;
#pragma unroll
                for (int i = 0; i < NV * Z::VE; i++) {
                    const bool in = k[i] != 0 && k[i] >= bound;
                    const uint64_t all = __ballot(in);
                    const int at = count + __builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32),
                                                                     __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0));
                    if (in && at < WAVE_LIST)
                        found[at] = k[i];
                    count += __popcll(all);
                }
                if (count <= WAVE_LIST) {
                    if (lane < 4 && count + lane < WAVE_LIST)
                        found[count + lane] = 0;
                    wave_fence();
                    for (int i = lane; i < count; i += 64) {
                        const Key one = found[i];
                        int rank = 0;
#pragma unroll 2
                        for (int j = 0; j < count; j += 4) {
                            struct __align__(16) Four {
                                Key k[4];
                            };
                            const Four o = *reinterpret_cast<const Four *>(found + j);
#pragma unroll
                            for (int u = 0; u < 4; u++)
                                rank += o.k[u] > one;
                        }
                        if (rank < a.top)
                            put_top(a, row, rank, K::wide(one), st);
                    }
                    from = a.top;
                }
            }
        for (int n = from; n < a.top; n++) {
            const typename K::key best = K::template best<G>(top);
            mine = n == lane ? best : mine;
            if (top == best) {
                top = 0;
#pragma unroll
                for (int i = 0; i < NV * Z::VE; i++)
                    top = k[i] < best && k[i] > top ? k[i] : top;
            }
        }
        if (from == 0 && lane < a.top)
            put_top(a, row, lane, K::wide(mine), st);
    }
    if (lane == 0)  // last: the asked logit is two loads, one after the other
        finish(a, row, st, asked);
}

constexpr int CHUNKS = 64;  // at most, one a lane of the joining wave

// The chunks of a row: a lane each; alternatives by merging their lists.
template <typename Z, bool TOP>
__global__ __launch_bounds__(64) void log_probs_join_kernel(Args a) {
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    const bool on = lane < a.chunks;
    const Asked asked = ask<Z>(a, row);
    Stat st = {-INFINITY, 0.0f, 0.0f};
    if (on) {
        const float4 p = a.part[row * a.chunks + lane];
        st = {p.x, p.y, p.z};
    }
    st = wave_join(st);
    if constexpr (TOP) {
        __shared__ uint64_t key[CHUNKS * TOP_MAX];
        const uint64_t *const from = a.part_key + row * a.chunks * a.top;
        // eight loads in flight
        for (int i = lane; i < a.chunks * a.top; i += 8 * 64) {
            uint64_t k[8];
#pragma unroll
            for (int u = 0; u < 8; u++)
                k[u] = i + u * 64 < a.chunks * a.top ? from[i + u * 64] : 0;
#pragma unroll
            for (int u = 0; u < 8; u++)
                if (i + u * 64 < CHUNKS * TOP_MAX)
                    key[i + u * 64] = k[u];
        }
        __syncthreads();
        int at = 0;
        uint64_t head = on ? key[lane * a.top] : 0, mine = 0;
        for (int n = 0; n < a.top; n++) {
            const uint64_t best = wave_max(head);
            if (n == lane)
                mine = best;
            if (head == best && best != 0) {
                at++;
                head = at < a.top ? key[lane * a.top + at] : 0;
            }
        }
        if (lane < a.top)
            put_top(a, row, lane, mine, st);
    }
    if (lane == 0)
        finish(a, row, st, asked);
}

// ---------------------------------------------------------------------------
struct BackArgs {
    const void *z;
    void *dz;
    const int64_t *tokens;
    const float2 *stats;
    const float *entropy, *d_logp, *d_entropy;
    int64_t ldz, lddz;
    int V;
    uint32_t n;       // vectors of all rows
    FastDiv per_row;  // vectors of a row
};

// What the vectors of a row share:  dz_j = p_j (a + b l_j), l_j = log2 p_j.
struct RowGrad {
    float ref, off, a, b, g;
    int64_t token;
};
__device__ __forceinline__ RowGrad row_grad(const BackArgs &k, int64_t row) {
    RowGrad r;
    const float2 st = k.stats[row];
    const bool bad = !(st.x < INFINITY), empty = st.x == -INFINITY;
    const float h = k.d_entropy ? k.d_entropy[row] : 0.0f;
    r.token = k.tokens ? k.tokens[row] : -1;
    r.g = r.token >= 0 && k.d_logp ? k.d_logp[row] : 0.0f;
    r.ref = ref_of(st.x);
    r.off = -st.y * LOG2E;
    r.a = k.d_entropy ? -r.g - h * k.entropy[row] : -r.g;
    r.b = -h * LN2;
    if (empty)
        r.a = r.b = r.g = 0.0f;
    if (bad || r.token >= k.V)  // no such class: the forward pass said NaN
        r.a = NAN;
    return r;
}

// n (at most a vector's) logits from index i on
template <typename Z>
__device__ __forceinline__ void grad8(const BackArgs &k, const RowGrad &r, const typename Z::elem *z,
                                      typename Z::elem *dz, int i, int n) {
    float x[Z::VE];
    Z::values(Z::load(z, i, k.V), n, x);
#pragma unroll
    for (int e = 0; e < Z::VE; e++) {
        const float l = fmaxf(fmaf(x[e] - r.ref, LOG2E, r.off), FLOOR2);
        x[e] = __builtin_amdgcn_exp2f(l) * fmaf(r.b, l, r.a);
    }
    if (r.token >= i && r.token < i + n)
#pragma unroll
        for (int e = 0; e < Z::VE; e++)
            if (r.token == i + e)
                x[e] += r.g;
    Z::store(dz, i, i + n, x);
}

// Short rows: a thread takes a vector of any row.
template <typename Z>
__global__ __launch_bounds__(256) void log_probs_backward_kernel(BackArgs k) {
    const uint32_t v = blockIdx.x * 256 + threadIdx.x;
    if (v >= k.n)
        return;
    const uint32_t row = fdiv(v, k.per_row);
    const int i = (int)(v - row * k.per_row.d) * Z::VE;
    grad8<Z>(k, row_grad(k, row), (const typename Z::elem *)k.z + row * k.ldz,
             (typename Z::elem *)k.dz + row * k.lddz, i, k.V - i);
}

// Long rows: a workgroup takes BACK_NV * 256 vectors of one row, whose numbers
// it reads once.
constexpr int BACK_NV = 4;
template <typename Z>
__global__ __launch_bounds__(256) void log_probs_backward_row_kernel(BackArgs k, uint32_t chunks) {
    const uint32_t row = blockIdx.x / chunks, part = blockIdx.x - row * chunks;
    const RowGrad r = row_grad(k, row);
    const typename Z::elem *const z = (const typename Z::elem *)k.z + row * k.ldz;
    typename Z::elem *const dz = (typename Z::elem *)k.dz + row * k.lddz;
    const Piece<Z> piece(z, 0, k.V, k.V);
#pragma unroll
    for (int u = 0; u < BACK_NV; u++) {
        const int v = (int)(part * BACK_NV + u) * 256 + (int)threadIdx.x;
        if (v < piece.vectors()) {
            const auto a = piece.at(v);
            grad8<Z>(k, r, z, dz, a.i, a.n);
        }
    }
}

// Chunks of a row, and their length: rows enough to fill the chip stay whole;
// otherwise about four workgroups a CU, of at least a vector for each thread.
void chunks_of(int64_t rows, int V, int *chunks, int *chunk) {
    int64_t n = (4 * device_cu_count() + rows - 1) / rows;
    const int64_t most = (V + 2047) / 2048;
    n = n < most ? n : most;
    n = n < CHUNKS ? n : CHUNKS;
    n = rows >= 2 * device_cu_count() || n < 1 ? 1 : n;
    *chunk = (int)((V + n - 1) / n + 7) / 8 * 8;
    *chunks = (V + *chunk - 1) / *chunk;
}

template <typename Z, int G, int N>
hipError_t forward_wave(const Args &a, int64_t rows, hipStream_t st) {
    const dim3 grid((unsigned)((rows + 256 / G - 1) / (256 / G)));
    if (a.top)
        log_probs_wave_kernel<Z, G, N, true><<<grid, dim3(256), 0, st>>>(a, rows);
    else
        log_probs_wave_kernel<Z, G, N, false><<<grid, dim3(256), 0, st>>>(a, rows);
    return hipGetLastError();
}

template <typename Z>
hipError_t forward(const Args &a, int64_t rows, hipStream_t st) {
    // a lane for each of the alternatives
    if (a.V <= 8 * Z::VE && a.top <= 8)
        return forward_wave<Z, 8, 1>(a, rows, st);
    if (a.V <= 16 * Z::VE && a.top <= 16)
        return forward_wave<Z, 16, 1>(a, rows, st);
    if (a.V <= 32 * Z::VE)
        return forward_wave<Z, 32, 1>(a, rows, st);
    if (a.V <= 64 * Z::VE)
        return forward_wave<Z, 64, 1>(a, rows, st);
    if (a.V <= 128 * Z::VE)
        return forward_wave<Z, 64, 2>(a, rows, st);
    // Longer rows with alternatives go to a wave each where that fills the card, to
    // a workgroup each (or several) where they are fewer.  bf16, eight: 100 rows of
    // 2000 7.3 us by workgroups, 8.3 by waves (twenty 7.6 and 15), 1000 9.0 and
    // 8.5; 500 rows of 4000 13.4 and 12.2 (twenty 16 and 19), 3000 24 and 19.
    const int64_t cus = device_cu_count();
    if (a.V <= 256 * Z::VE && (a.top <= 4 || rows >= 4 * cus))
        return forward_wave<Z, 64, 4>(a, rows, st);
    if (a.V <= 512 * Z::VE && (a.top == 0 || rows >= 4 * cus))
        return forward_wave<Z, 64, 8>(a, rows, st);
    const dim3 grid((unsigned)(rows * a.chunks));
    // Short chunks, few vectors a thread: less code for what runs once (one row of
    // 131072 with eight alternatives 9.7 us a call, 9.9 with four vectors; 32 of
    // 50257 with twenty 15.1 and 16.7).
    if (a.chunk <= 2048)
        a.top ? log_probs_kernel<Z, true, 1><<<grid, dim3(TH), 0, st>>>(a)
              : log_probs_kernel<Z, false, 1><<<grid, dim3(TH), 0, st>>>(a);
    else
        a.top ? log_probs_kernel<Z, true, 4><<<grid, dim3(TH), 0, st>>>(a)
              : log_probs_kernel<Z, false, 4><<<grid, dim3(TH), 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.chunks == 1)
        return e;
    if (a.top)
        log_probs_join_kernel<Z, true><<<dim3((unsigned)rows), dim3(64), 0, st>>>(a);
    else
        log_probs_join_kernel<Z, false><<<dim3((unsigned)rows), dim3(64), 0, st>>>(a);
    return hipGetLastError();
}

// Workgroups of a row of the backward pass (0: a short one); `size` bytes a logit.
uint32_t back_chunks(const void *z, int64_t ldz, int V, int size) {
    const int ve = 16 / size, span = BACK_NV * 256 * ve;
    if (V < span / 2)
        return 0;
    // room for a first vector that is not whole, unless every row starts a vector
    const bool whole = ((uintptr_t)z | (uintptr_t)ldz * size) % 16 == 0;
    return (uint32_t)(((int64_t)V + (whole ? 0 : ve - 1) + span - 1) / span);
}

template <typename Z>
hipError_t backward(BackArgs &a, int64_t rows, hipStream_t st) {
    if (const uint32_t chunks = back_chunks(a.z, a.ldz, a.V, sizeof(typename Z::elem))) {
        log_probs_backward_row_kernel<Z><<<dim3((unsigned)(rows * chunks)), dim3(256), 0, st>>>(a, chunks);
    } else {
        const uint32_t per_row = (uint32_t)((a.V + Z::VE - 1) / Z::VE);
        a.per_row = make_fastdiv(per_row);
        a.n = (uint32_t)(rows * per_row);
        log_probs_backward_kernel<Z><<<dim3((a.n + 255) / 256), dim3(256), 0, st>>>(a);
    }
    return hipGetLastError();
}

size_t keys_at(int64_t rows, int chunks) { return (size_t)rows * chunks * sizeof(float4); }

}  // namespace

// Grids stay below 2^32 threads, vectors of short rows below 2^31.
bool log_probs_fit(int64_t rows, int V) {
    const double limit = 16777216.0;
    return rows < limit && (V >= 4096 ? (double)rows * ((V + 4095) / 4096) < limit
                                      : (double)rows * ((V + 3) / 4) < 2147483648.0);
}

bool log_probs_backward_fits(const LogProbsBackward &p, int64_t rows, int V, int dt) {
    const uint32_t chunks = back_chunks(p.z, p.ldz, V, dt == LOGITS_F32 ? 4 : 2);
    return log_probs_fit(rows, V) && (double)rows * chunks < 16777216.0;
}

size_t log_probs_workspace_bytes(int64_t rows, int V, int top) {
    int chunks, chunk;
    chunks_of(rows, V, &chunks, &chunk);
    return chunks > 1 ? keys_at(rows, chunks) + (size_t)rows * chunks * top * sizeof(uint64_t) : 0;
}

hipError_t launch_log_probs(const LogProbs &p, int64_t rows, int V, int top, int dt, void *ws, hipStream_t st) {
    Args a;
    a.z = p.z;
    a.tokens = p.tokens;
    a.logp = p.logp;
    a.entropy = p.entropy;
    a.stats = (float2 *)p.stats;
    a.top_logp = p.top_logp;
    a.top_ids = p.top_ids;
    a.ldz = p.ldz;
    a.V = V;
    a.top = top;
    chunks_of(rows, V, &a.chunks, &a.chunk);
    a.part = (float4 *)ws;
    a.part_key = (uint64_t *)((char *)ws + keys_at(rows, a.chunks));
    return dt == LOGITS_F32 ? forward<Z32>(a, rows, st)
           : dt == LOGITS_BF16 ? forward<Z16<BF16>>(a, rows, st)
                               : forward<Z16<F16>>(a, rows, st);
}

hipError_t launch_log_probs_backward(const LogProbsBackward &p, int64_t rows, int V, int dt, hipStream_t st) {
    BackArgs a;
    a.z = p.z;
    a.dz = p.dz;
    a.tokens = p.tokens;
    a.stats = (const float2 *)p.stats;
    a.entropy = p.entropy;
    a.d_logp = p.d_logp;
    a.d_entropy = p.d_entropy;
    a.ldz = p.ldz;
    a.lddz = p.lddz;
    a.V = V;
    a.n = 0;
    a.per_row = FastDiv{1, 0, 0};
    return dt == LOGITS_F32 ? backward<Z32>(a, rows, st)
           : dt == LOGITS_BF16 ? backward<Z16<BF16>>(a, rows, st)
                               : backward<Z16<F16>>(a, rows, st);
}

}  // namespace cf
