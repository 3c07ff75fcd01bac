// Attention for trees of drafted tokens over the paged K/V cache, and the weight that cached tokens get from it.
//
// Request i has L_i context tokens in the pool and a tree of n_i <= 64 nodes: node 0 is the pending token, node j continues node
// parent[j] < j.  A node sees the whole context, its ancestors and itself; which nodes those are is one 64-bit word per node.
// With A(j) the ancestors of j and j itself, for query head h of kv head g = h / G:
//   s_t = q_jh . K_gt / sqrt(D)   (t < L, and the nodes t in A(j))
//   lse = log sum exp(s_t),   out = sum exp(s_t - lse) V_gt
//
// tree_attention_kernel, per work item (request, kv head, group of stacked rows, run of context pages):
//   All G heads of all nodes are stacked into tiles of 16 rows (row r = node r / G, head r % G), so that K and V are read from memory once for up to
//   128 rows.  The eight wavefronts of a workgroup, one workgroup a CU, read a step's K and V (32 tokens: two pages) together, 16 bytes a lane, into
//   registers, 64 KB ahead, and hand them over through LDS in the order the products want them.  Each has one row tile; with no more
//   than four (two) tiles, two (four) groups of wavefronts take a step each.
//     S^T[32 tokens, 16 rows] = K Q^T    v_mfma_f32_16x16x32_bf16, page by page
//     O^T[128 dims, 16 rows] += V^T P^T  the same instruction over both pages at once: a lane holds, of S^T, the four tokens of its
//                                        quad in each page, and these eight are its part of the operand P^T, as the quads of V are of V^T
//   p = 2^(s' - M), s' in log2 units, M a whole number that a row raises when some s' passes it by more than 16; every rescale is then an
//   exact power of two, so neither the order of the pages nor their split over wavefronts changes how p is rounded.  p enters the second product as
//   a bf16 pair (16 bits), which costs 8 of 24 instructions: with a single bf16 the error would be that of the output's own
//   rounding once more.  Sums are float32.
//   The tree's own keys and values come from the caller's k and v as one or two more steps under the ancestors' bits; the item that reads them also
//   writes them into the request's tail slots, which nobody reads in this launch.  Items of one (request, kv head, row group) store their
//   states and the last to arrive adds them up in ascending order.
//   fp32 models: the same with v_mfma_f32_16x16x4_f32 and single pages.
// What bounds it: a step of 32 tokens costs a wavefront 24 matrix instructions, 85 vector ones and 8 exponentials.  On one SIMD matrix instructions hold
// the port for 8 clocks, the others for 4 to 5 and exponentials for 9 (measured), so two wavefronts need 1200 clocks a step where 1650 are measured; the
// rest is the wait at the step's barrier and for LDS.  16 requests (982 pages, 84 rows each, 8 kv heads) take 29 us a layer, 77 MB fetched
// and 14 written; 64 requests (7204 pages, 139 rows each) 164 us with 566 to 592 MB fetched (472 without what second row groups read again) and
// 66 written (27 of them results), 4.0 TB/s; one request of 300 tokens 9.9 us, a chain of launch, item, pages, three turns of LDS and
// memory latency, merge.  Tried: DMA into LDS (a wavefront is held 200 clocks for each), wavefronts that read their own steps from memory (every row tile
// of a wavefront costs registers, 128 rows need two: 200 us), K read a step early over a third LDS buffer (198 us), two steps between
// barriers (188 us), all wavefronts in phase (174 us).
// A value that is not finite must not reach the rows that do not see its node (0 * inf is NaN): such values of v are left out of the
// product and added at the end for the rows that do see them.  Slots of the last context page behind L count as zero.
#include "sled_internal.h"

#include <type_traits>

namespace {

constexpr float NEG_BIG = -1.0e30f;
constexpr int WAVES = 8;

// (vectors of the compiler's own: structs of four would not stay in registers where their parts are used)
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// sizes of one step of the page loop
template <int D, bool F32>
struct Geo {
    static constexpr int P = F32 ? 1 : 2;        // pages
    static constexpr int TOK = 16 * P;           // tokens
    static constexpr int DT = D / 16;            // tiles of 16 dims of an output
    static constexpr int QC = F32 ? D / 16 : 4;  // operand pieces (16 bytes a lane) of a row tile, per plane
    static constexpr int ELEM = F32 ? 4 : 2;
    static constexpr int CH = D * ELEM / 16;     // 16-byte pieces of a token
    static constexpr int BYTES = TOK * D * ELEM; // of K or of V
    static constexpr int LOADS = 2 * BYTES / (64 * WAVES * 16);   // pieces that a thread moves: one of K and one of V, or (1) the upper half of the threads V
};

// one step's K, and its V with the weights it is to be multiplied by, as the lanes hold them
template <int D, bool F32>
struct Keys {
    u32x4 k[2][4];   // [page][32 dims]: token lane % 16, dims (lane / 16) * 8 ..
};
template <int D>
struct Keys<D, true> {
    f32x4 k[D / 16];   // token lane % 16, dims 16 c + (lane / 16) * 4 ..
};
template <int D, bool F32>
struct Values {
    u32x4 v[8];      // [16 dims]: tokens (lane / 16) * 4 .. + 3 of dim lane % 16, of the first page and of the second
    u32x4 hi, lo;    // weights of these tokens for row lane % 16
};
template <int D>
struct Values<D, true> {
    float v[D / 16][4];   // token (lane / 16) * 4 + i, dim 16 dt + lane % 16
    float w[4];
};

// A step in LDS: K, then V.  bf16: K pages as they are in the pool, V as the operands of its eight tiles of dims.  fp32: K as [16 dims][lane] pieces
// of 16 bytes, V as rows whose runs of 16 dims are turned by token / 4 places within their four: lane groups read tokens four
// apart and so meet different banks.
__device__ __forceinline__ int turned(int t, int q) { return (q & ~15) | ((q + (t >> 2) * 4) & 12) | (q & 3); }

template <int D, bool F32>
__device__ __forceinline__ void read_keys(Keys<D, F32>& kv, const char* step, int lane) {
    const u32x4* k = reinterpret_cast<const u32x4*>(step) + lane;
    if constexpr (!F32) {
#pragma unroll
        for (int p = 0; p < 2; p++)
#pragma unroll
            for (int c = 0; c < 4; c++) kv.k[p][c] = k[p * 256 + c * 64];
    } else {
#pragma unroll
        for (int c = 0; c < D / 16; c++) kv.k[c] = __builtin_bit_cast(f32x4, k[c * 64]);
    }
}
template <int D, bool F32>
__device__ __forceinline__ void read_values(Values<D, F32>& kv, const char* step, int lane) {
    if constexpr (!F32) {
        const u32x4* v = reinterpret_cast<const u32x4*>(step + Geo<D, F32>::BYTES) + lane;
#pragma unroll
        for (int dt = 0; dt < 8; dt++) kv.v[dt] = v[dt * 64];
    } else {
        const float* v = reinterpret_cast<const float*>(step + Geo<D, F32>::BYTES) + (lane >> 4) * 4 * D + (lane & 15);
#pragma unroll
        for (int dt = 0; dt < D / 16; dt++)
#pragma unroll
            for (int i = 0; i < 4; i++) kv.v[dt][i] = v[i * D + ((dt & ~3) | ((dt + (lane >> 4)) & 3)) * 16];
    }
}

// this thread's share of a step on its way to LDS
template <int D, bool F32>
struct Cargo {
    u32x4 x[Geo<D, F32>::LOADS];
};
template <int D, bool F32>
__device__ __forceinline__ bool is_value(int u, int wave) {
    return Geo<D, F32>::LOADS == 2 ? u == 1 : wave >= WAVES / 2;
}

// values of tokens lim .. count as zero; e: the piece's number among those of V
template <int D, bool F32>
__device__ __forceinline__ void cut_values(u32x4& x, int lim, int e) {
    if constexpr (F32) {
        if (e / Geo<D, F32>::CH >= lim) x = u32x4{0u, 0u, 0u, 0u};
    } else {
        const int t = (e >> 8) * 16 + ((e >> 4) & 3) * 4;   // the piece holds tokens t .. t + 3 of two dims
        const uint32_t a = (t < lim ? 0xffffu : 0u) | (t + 1 < lim ? 0xffff0000u : 0u), b = (t + 2 < lim ? 0xffffu : 0u) | (t + 3 < lim ? 0xffff0000u : 0u);
        x &= u32x4{a, b, a, b};
    }
}

// piece e of K or V of context pages
template <int D, bool F32>
__device__ __forceinline__ void store_piece(const u32x4& x, bool value, int e, char* step) {
    constexpr int CH = Geo<D, F32>::CH;
    if constexpr (F32) {
        const int t = e / CH, q = e % CH;
        if (value) reinterpret_cast<u32x4*>(step + Geo<D, F32>::BYTES)[t * CH + turned(t, q)] = x;
        else reinterpret_cast<u32x4*>(step)[(q >> 2) * 64 + (q & 3) * 16 + t] = x;
    } else if (value) {
        // 8 bytes of each of two operands
        u32x2* v = reinterpret_cast<u32x2*>(step + 8192) + (((e & 255) >> 6) * 128 + (e & 63)) * 2 + (e >> 8);
        v[0] = u32x2{x[0], x[1]};
        v[128] = u32x2{x[2], x[3]};
    } else {
        reinterpret_cast<u32x4*>(step)[e] = x;
    }
}

__device__ __forceinline__ float max_over_groups(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_over_groups(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// S of a row tile against one page (A operand Q, B operand K)
template <int D, bool F32, int PL>
__device__ __forceinline__ float4_t page_scores(const Keys<D, F32>& kv, int sub, const u32x4* q /* the tile's operand pieces + lane */) {
    float4_t s = {0.f, 0.f, 0.f, 0.f};
    if constexpr (!F32) {
#pragma unroll
        for (int ks = 0; ks < 4; ks++)
#pragma unroll
            for (int pl = 0; pl < PL; pl++)
                s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, q[(pl * 4 + ks) * 64]), __builtin_bit_cast(bf16x8_t, kv.k[sub][ks]), s, 0, 0, 0);
    } else {
#pragma unroll
        for (int c = 0; c < D / 16; c++) {
            const f32x4 kk = kv.k[c], xx = __builtin_bit_cast(f32x4, q[c * 64]);
#pragma unroll
            for (int e = 0; e < 4; e++) s = __builtin_amdgcn_mfma_f32_16x16x4f32(xx[e], kk[e], s, 0, 0, 0);
        }
    }
    return s;
}

// where the operand piece of row r (of its tile), 16 bytes number c of the row, sits among a tile's pieces of one plane
template <bool F32>
__device__ __forceinline__ int q_piece(int r, int c) {
    return (c >> 2) * 64 + (c & 3) * 16 + r;
}

struct tree_args {
    sled_tree_plan t;
    const int32_t* len_dev;
    const void* q;             // rows of n_q_heads * D, q_stride elements apart
    size_t q_stride, q_plane;  // PAIR: distance of the low plane
    const void *k, *v;         // rows of n_kv_heads * D, k_stride and v_stride elements apart
    size_t k_stride, v_stride;
    void *k_pool, *v_pool;
    int64_t n_pages;
    int layer, Hq, Hkv;
    float scale_log2;
    void* out;                 // rows of n_q_heads * D; STEP and bf16: operand order of the following projection, two planes
    size_t x_plane;
    float* lse;                // or nullptr
};

// Rows r0 .. r0 + n_rows - 1 of a block's stacked rows on their way into LDS, as the operand pieces of their tiles: a thread's pieces e0, e0 + nt, ...
template <int D, bool F32, int PL, int N>
__device__ __forceinline__ void ask_queries(u32x4 (&x)[N], const tree_args& a, int row0, int g, int G, int r0, int rows, int e0, int nt) {
    constexpr int CH = D * Geo<D, F32>::ELEM / 16;   // 16-byte pieces of a row
    asm volatile("" : "+v"(e0));   // (addresses are made when they are needed: kept, they would cost registers)
#pragma unroll
    for (int u = 0; u < N; u++) {
        const int e = e0 + u * nt, c = e % CH, pl = e / CH % PL, r = min(r0 + e / (CH * PL), rows - 1);   // (any row that there is)
        const int j = r / G, hh = r - j * G;
        const size_t at = (pl * a.q_plane + (size_t)(row0 + j) * a.q_stride + (size_t)(g * G + hh) * D) * Geo<D, F32>::ELEM + c * 16;
        x[u] = *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.q) + at);
    }
}
// ... and there; rows from `rows` on are zero
template <int D, bool F32, int PL, int N>
__device__ __forceinline__ void put_queries(u32x4* qs, const u32x4 (&x)[N], int r0, int n_rows, int rows, int e0, int nt) {
    constexpr int CH = D * Geo<D, F32>::ELEM / 16;
    asm volatile("" : "+v"(e0));
#pragma unroll
    for (int u = 0; u < N; u++) {
        const int e = e0 + u * nt, c = e % CH, pl = e / CH % PL, rr = e / (CH * PL);
        if (rr < n_rows) qs[((rr >> 4) * PL + pl) * CH * 16 + q_piece<F32>(rr & 15, c)] = r0 + rr < rows ? x[u] : u32x4{0u, 0u, 0u, 0u};
    }
}

// The running state of a wavefront: row lane % 16 of its tile, dims 16 dt + (lane / 16) * 4 + e
template <int DT>
struct State {
    float m, l;   // reference; this lane's part of the sum
    float4_t o[DT];
};

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Scores of a step against the wavefront's row tile, their weights, and V on its way.  MASKED: bit t of `bits` says whether this lane's row sees token t.
template <int D, bool F32, int PL, bool MASKED>
__device__ __forceinline__ void weigh(const char* step, const u32x4* q, int lane, float c, uint32_t bits, State<D / 16>& st, Values<D, F32>& x_v) {
    constexpr int P = Geo<D, F32>::P, DT = Geo<D, F32>::DT;
    const int t0 = (lane >> 4) * 4;
    Keys<D, F32> kv;
    read_keys<D, F32>(kv, step, lane);
    read_values<D, F32>(x_v, step, lane);
    __builtin_amdgcn_sched_barrier(0);   // (V is on its way while the scores are made)
    float4_t s[P];
#pragma unroll
    for (int p = 0; p < P; p++) s[p] = float4_t{0.f, 0.f, 0.f, 0.f};
    if constexpr (!F32) {
#pragma unroll
        for (int ks = 0; ks < 4; ks++)
#pragma unroll
            for (int pl = 0; pl < PL; pl++)
#pragma unroll
                for (int p = 0; p < P; p++)
                    s[p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kv.k[p][ks]), __builtin_bit_cast(bf16x8_t, q[pl * 4 + ks]), s[p], 0, 0, 0);
    } else {
#pragma unroll
        for (int d = 0; d < D / 16; d++) {
            const f32x4 kk = kv.k[d], xx = __builtin_bit_cast(f32x4, q[d]);
#pragma unroll
            for (int e = 0; e < 4; e++) s[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(kk[e], xx[e], s[0], 0, 0, 0);
        }
    }
    if (MASKED) {
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int i = 0; i < 4; i++) s[p][i] = (bits >> (p * 16 + t0 + i)) & 1u ? s[p][i] : -INFINITY;
    }
    float x[P * 4], top = -INFINITY;
#pragma unroll
    for (int p = 0; p < P; p++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
            x[p * 4 + i] = fmaf(s[p][i], c, -st.m);
            top = fmaxf(top, x[p * 4 + i]);
        }
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(top > 16.f) != 0ull, 0)) {
        // some row's reference is too low: raise it to a whole number (row by row; the four lanes of a row agree)
        float hi = s[0][0];
#pragma unroll
        for (int i = 1; i < P * 4; i++) hi = fmaxf(hi, s[i >> 2][i & 3]);
        const float mnew = fmaxf(st.m, ceilf(max_over_groups(hi) * c)), alpha = __builtin_amdgcn_exp2f(st.m - mnew);
        st.m = mnew;
        st.l *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; dt++)
#pragma unroll
            for (int e = 0; e < 4; e++) st.o[dt][e] *= alpha;
#pragma unroll
        for (int i = 0; i < P * 4; i++) x[i] = fmaf(s[i >> 2][i & 3], c, -st.m);
    }
    float w[P * 4];
#pragma unroll
    for (int i = 0; i < P * 4; i++) w[i] = __builtin_amdgcn_exp2f(x[i]);
    if constexpr (!F32) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            x_v.hi[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{w[2 * i], w[2 * i + 1]}), bf16x2));   // to nearest even
            const float r0 = w[2 * i] - __uint_as_float(x_v.hi[i] << 16), r1 = w[2 * i + 1] - __uint_as_float(x_v.hi[i] & 0xffff0000u);
            x_v.lo[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{r0, r1}), bf16x2));
        }
        st.l += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) x_v.w[i] = w[i];
        st.l += (w[0] + w[1]) + (w[2] + w[3]);
    }
}

template <int D, bool F32>
__device__ __forceinline__ void gather(const Values<D, F32>& x, State<D / 16>& st) {
    constexpr int DT = D / 16;
    if constexpr (!F32) {
        const bf16x8_t ph = __builtin_bit_cast(bf16x8_t, x.hi), pl = __builtin_bit_cast(bf16x8_t, x.lo);
#pragma unroll
        for (int dt = 0; dt < DT; dt++) st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x.v[dt]), ph, st.o[dt], 0, 0, 0);
#pragma unroll
        for (int dt = 0; dt < DT; dt++) st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x.v[dt]), pl, st.o[dt], 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int dt = 0; dt < DT; dt++) st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.v[dt][i], x.w[i], st.o[dt], 0, 0, 0);
    }
}

__device__ __forceinline__ bool not_finite(bf16_t x) { return (x & 0x7f80) == 0x7f80; }
__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

// of 16 bytes of values: whether one of them is not finite (an exponent of ones), and the others alone
template <bool F32>
__device__ __forceinline__ bool has_not_finite(const u32x4& v) {
    constexpr uint32_t EXP = F32 ? 0x7f800000u : 0x7f807f80u, ONE = F32 ? 0x00800000u : 0x00800080u, TOP = F32 ? 0x80000000u : 0x80008000u;
    uint32_t over = 0u;
#pragma unroll
    for (int i = 0; i < 4; i++) over |= (v[i] & EXP) + ONE;   // the exponent of ones carries into the sign's place
    return (over & TOP) != 0u;
}
template <bool F32>
__device__ __forceinline__ u32x4 finite_only(u32x4 v) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if constexpr (F32) {
            if ((v[i] & 0x7f800000u) == 0x7f800000u) v[i] = 0u;
        } else {
            if ((v[i] & 0x7f80u) == 0x7f80u) v[i] &= 0xffff0000u;
            if ((v[i] & 0x7f800000u) == 0x7f800000u) v[i] &= 0xffffu;
        }
    }
    return v;
}

// register i of lane group g <-> register g of lane group i
__device__ __forceinline__ void quad_transpose(u32x4& v) {
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const auto x = __builtin_amdgcn_permlane32_swap(v[i], v[i + 2], false, false);
        v[i] = x[0];
        v[i + 2] = x[1];
    }
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const auto x = __builtin_amdgcn_permlane16_swap(v[i], v[i + 1], false, false);
        v[i] = x[0];
        v[i + 1] = x[1];
    }
}

// bytes of LDS: two steps of every token group; afterwards the states that the token groups exchange
template <int NR, int D, bool F32>
constexpr size_t attention_lds() {
    constexpr size_t NG = WAVES / NR, loop = 2 * NG * 2 * Geo<D, F32>::BYTES, merge = NG > 1 ? (size_t)WAVES * Geo<D, F32>::DT * 1024 : 0;
    return loop > merge ? loop : merge;
}

// LDS beside the steps
struct tree_shared {
    int pages[SLED_TREE_RUN];
    float m[WAVES * 16], l[WAVES * 16];   // [token group][row]
    uint32_t bad[2];                      // nodes with values that are not finite
    int last;
};

// NR wavefronts share the row tiles (one each), WAVES / NR groups of wavefronts share the steps
template <int NR, int D, bool F32, bool STEP>
__device__ __forceinline__ void attend_item(const tree_args& a, const int32_t* rec, unsigned char* smem, tree_shared& sh) {
    using G_ = Geo<D, F32>;
    using T = std::conditional_t<F32, float, bf16_t>;
    constexpr int NG = WAVES / NR, ROWS = NR * 16, DEPTH = 4 / NG;   // token groups; turns asked for ahead
    constexpr int P = G_::P, TOK = G_::TOK, DT = G_::DT, OWN = DT / NG, PL = STEP && !F32 ? 2 : 1, LOADS = G_::LOADS, CH = G_::CH, E = 16 / G_::ELEM;
    const int w = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int req = rec[0], g = rec[1], page0 = rec[2], npg = rec[3], n = rec[4], row0 = rec[5], w0 = rec[7], n_items = rec[8], stride = rec[9], r0 = rec[10];
    const bool last = rec[11] != 0;   // the item that has the tree
    const int n_tiles = rec[12], slot0 = rec[14];
    const int32_t* pages = a.t.pages + rec[6];
    for (int i = tid; i < max(npg, 1); i += 64 * WAVES) sh.pages[i] = pages[page0 + i];   // (without context: the request's first page)
    const int L = a.len_dev[req];
    const int G = a.Hq / a.Hkv;
    const int rw = wave % NR, tg = wave / NR, lr = lane & 15, lg = lane >> 4;
    const bool mine = rw < n_tiles;   // this wavefront has a tile
    const size_t head = (size_t)16 * D, layer_page = (size_t)a.layer * a.n_pages;

    // the item's steps: its pages, as far as there is context, then the tree's
    const int n_pages = max(0, min(npg, ((L + 15) >> 4) - page0)), n_ctx = (n_pages + P - 1) / P;
    const int n_sub = n_ctx + (last ? (n + TOK - 1) / TOK : 0), n_turns = (n_sub + NG - 1) / NG;
    const int n_full = max(0, min(L - page0 * 16, n_pages * 16)) / TOK / (NG * DEPTH) * DEPTH;   // turns, in rounds of DEPTH, without a mask
    if (tid < 2) sh.bad[tid] = 0u;
    __syncthreads();

    // Turns on their way, DEPTH of them.  Every request is made, whatever the turn: one behind the last step asks for one line again.  So the number
    // of requests behind the one that is waited for is always the same, and nothing else has to be waited for.
    Cargo<D, F32> cargo[DEPTH][NG];
    const int half = (F32 ? 0 : wave >> 2);   // which of the step's pages this wavefront's pieces belong to
    const int e = LOADS == 2 ? tid : tid & (32 * WAVES - 1);   // the thread's piece of K or V
    const char* k_base = static_cast<const char*>(a.k_pool) + (layer_page * a.Hkv + g) * head * G_::ELEM;
    const char* v_base = static_cast<const char*>(a.v_pool) + (layer_page * a.Hkv + g) * head * G_::ELEM;
    const uint32_t page_bytes = (uint32_t)(a.Hkv * head * G_::ELEM), lane_off = (F32 ? e : tid & 255) * 16;
    int ids[NG];   // pages of the next request: read from LDS a turn before they are needed
    auto next_ids = [&](int s) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NG; u++) ids[u] = sh.pages[max(0, min(P * (s * NG + u) + half, n_pages - 1))];   // (any page that there is)
    };
    auto load = [&](Cargo<D, F32>* to, int s) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NG; u++) {
            const int i = s * NG + u;
            const uint64_t at = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane(ids[u]) * page_bytes;
            if (i < n_ctx || i >= n_sub) {
#pragma unroll
                for (int x = 0; x < LOADS; x++) to[u].x[x] = *reinterpret_cast<const u32x4*>((is_value<D, F32>(x, wave) ? v_base : k_base) + at + lane_off);
            } else {
                const size_t j = row0 + min((i - n_ctx) * TOK + e / CH, n - 1);
#pragma unroll
                for (int x = 0; x < LOADS; x++) {
                    const bool value = is_value<D, F32>(x, wave);
                    to[u].x[x] = *reinterpret_cast<const u32x4*>(static_cast<const char*>(value ? a.v : a.k) + (j * (value ? a.v_stride : a.k_stride) + g * D) * G_::ELEM + e % CH * 16);
                }
            }
        }
        asm volatile("" ::: "memory");   // asked for here, not where it is needed
        next_ids(s + 1);
    };
    auto step_at = [&](int s, int u) __attribute__((always_inline)) { return reinterpret_cast<char*>(smem) + ((s & 1) * NG + u) * 2 * G_::BYTES; };
    auto store = [&](Cargo<D, F32>* from, int s, auto masked) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NG; u++) {
            const int i = s * NG + u;
            char* to = step_at(s, u);
            if (!masked || i < n_ctx) {
                const int lim = L - (page0 + i * P) * 16;   // context tokens from the step's first on
#pragma unroll
                for (int x = 0; x < LOADS; x++) {
                    const bool value = is_value<D, F32>(x, wave);
                    if (masked && value && lim < TOK) cut_values<D, F32>(from[u].x[x], lim, e);
                    store_piece<D, F32>(from[u].x[x], value, e, to);
                }
            } else if (i < n_sub) {
                // nodes: rows of the caller's, their values turned here
#pragma unroll
                for (int x = 0; x < LOADS; x++) {
                    const bool value = is_value<D, F32>(x, wave);
                    const int t = e / CH, c = e % CH, j = (i - n_ctx) * TOK + t;
                    if (!value) {
                        if constexpr (F32) reinterpret_cast<u32x4*>(to)[(c >> 2) * 64 + (c & 3) * 16 + t] = from[u].x[x];
                        else *reinterpret_cast<u32x4*>(to + (t >> 4) * 4096 + kpage_offset(t & 15, c * 8) * 2) = from[u].x[x];
                        continue;
                    }
                    u32x4 v = from[u].x[x];
                    if (has_not_finite<F32>(v)) {
                        if (j < n) atomicOr(&sh.bad[j >> 5], 1u << (j & 31));
                        v = finite_only<F32>(v);
                    }
                    // (nodes behind the last repeat it: finite, and their weights are zero)
                    if constexpr (F32) {
                        reinterpret_cast<u32x4*>(to + G_::BYTES)[t * CH + turned(t, c)] = v;
                    } else {
                        // The wavefront has a token quad: lane group x token x, two dims a register.  Turned about its diagonal, a lane group has two
                        // dims of every token.
                        quad_transpose(v);
                        const int d = c * 8 + lg * 2;
                        u32x2* dst = reinterpret_cast<u32x2*>(to + G_::BYTES) + ((d >> 4) * 64 + ((t & 15) >> 2) * 16 + (d & 15)) * 2 + (t >> 4);
                        dst[0] = u32x2{(v[0] & 0xffffu) | (v[1] << 16), (v[2] & 0xffffu) | (v[3] << 16)};
                        dst[2] = u32x2{(v[0] >> 16) | (v[1] & 0xffff0000u), (v[2] >> 16) | (v[3] & 0xffff0000u)};
                    }
                }
            }
        }
    };

    // queries, in operand order: row lr of the wavefront's tile, 16 bytes number c
    u32x4 q[G_::QC * PL];
    const int r = r0 + rw * 16 + lr, node = mine ? r / G : n;   // this lane's row's node; n and beyond: none
    const int hh = r - r / G * G;
#pragma unroll
    for (int c = 0; c < G_::QC * PL; c++) {
        q[c] = u32x4{0u, 0u, 0u, 0u};
        if (node < n)
            q[c] = *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.q) +
                                                      ((c / G_::QC) * a.q_plane + (size_t)(row0 + node) * a.q_stride + (size_t)(g * G + hh) * D) * G_::ELEM +
                                                      (c % G_::QC * 4 + lg) * 16);
    }
    const uint64_t seen = node < n ? a.t.seen[row0 + node] : 0ull;
    next_ids(0);
#pragma unroll
    for (int u = 0; u < DEPTH; u++) load(cargo[u], u);

    State<DT> st;
    st.m = NEG_BIG;
    st.l = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; dt++) st.o[dt] = float4_t{0.f, 0.f, 0.f, 0.f};
    // The two wavefronts of a SIMD take turns: the upper four make their second product while the lower four make their scores, so that one's
    // matrix instructions run beside the other's exponentials.  (Wavefronts without a tile work on zeros: they would only wait otherwise.)
    Values<D, F32> held{};
    const bool late = wave >= WAVES / 2;
    auto turn = [&](Cargo<D, F32>* next, int s, auto masked) __attribute__((always_inline)) {
        // Into the buffer that everybody has read two turns ago; then the next request.  (A barrier for LDS alone: __syncthreads would
        // wait for the requests too.)
        store(next, s, masked);
        if (!masked || s + DEPTH < n_turns) load(next, s + DEPTH);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const int i = s * NG + tg;
        const char* step = step_at(s, tg);
        if (late) gather<D, F32>(held, st);
        if constexpr (!masked) {
            weigh<D, F32, PL, false>(step, q, lane, a.scale_log2, 0u, st, held);
        } else if (i < n_sub) {
            const int lim = L - (page0 + i * P) * 16;
            const uint32_t bits = i >= n_ctx ? (uint32_t)(seen >> ((i - n_ctx) * TOK)) : lim >= TOK ? ~0u : (1u << lim) - 1u;
            weigh<D, F32, PL, true>(step, q, lane, a.scale_log2, bits, st, held);
        } else {
            held = Values<D, F32>{};
        }
        if (!late) gather<D, F32>(held, st);
    };
    for (int s = 0; s < n_full; s += DEPTH) {
#pragma unroll
        for (int u = 0; u < DEPTH; u++) turn(cargo[u], s + u, std::false_type{});
    }
    if (n_full < n_turns)
        for (int s = n_full;;) {   // (left from the middle)
            turn(cargo[0], s, std::true_type{});
            if (++s >= n_turns) break;
            if constexpr (DEPTH >= 2) {
                turn(cargo[1], s, std::true_type{});
                if (++s >= n_turns) break;
            }
            if constexpr (DEPTH == 4) {
                turn(cargo[2], s, std::true_type{});
                if (++s >= n_turns) break;
                turn(cargo[3], s, std::true_type{});
                if (++s >= n_turns) break;
            }
        }
    if (late) gather<D, F32>(held, st);
    __syncthreads();   // nobody reads a step any more, and sh.bad is complete

    // sums over the lanes of a row
    float m = st.m, lsum = sum_over_groups(st.l);
    float4_t own[OWN];
    if constexpr (NG == 1) {
#pragma unroll
        for (int i = 0; i < OWN; i++) own[i] = st.o[i];
    } else {
        // token groups: each ends up with OWN of the dims' tiles of all of them, added in ascending order
        float* park = reinterpret_cast<float*>(smem);
        if (lg == 0) {
            sh.m[tg * ROWS + rw * 16 + lr] = m;
            sh.l[tg * ROWS + rw * 16 + lr] = lsum;
        }
#pragma unroll
        for (int dt = 0; dt < DT; dt++) *reinterpret_cast<float4_t*>(park + ((wave * DT + dt) * 64 + lane) * 4) = st.o[dt];
        __syncthreads();
        float im[NG];
#pragma unroll
        for (int u = 0; u < NG; u++) {
            im[u] = sh.m[u * ROWS + rw * 16 + lr];
            m = fmaxf(m, im[u]);
        }
        lsum = 0.f;
#pragma unroll
        for (int i = 0; i < OWN; i++) own[i] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < NG; u++) {
            const float f = exp2f(im[u] - m);
            lsum += sh.l[u * ROWS + rw * 16 + lr] * f;
#pragma unroll
            for (int i = 0; i < OWN; i++) own[i] += *reinterpret_cast<const float4_t*>(park + (((u * NR + rw) * DT + tg * OWN + i) * 64 + lane) * 4) * f;
        }
    }
    const int dt0 = tg * OWN;   // the first tile of dims that this wavefront has

    // The nodes' keys and values into the request's tail slots, which nobody reads in this launch: the last thing a workgroup does.  A thread takes
    // 16 bytes of the four tokens that V keeps together in a page.
    auto store_nodes = [&]() __attribute__((always_inline)) {
        const int quad0 = L >> 2, quads = ((L + n + 3) >> 2) - quad0;
        for (int e = tid; e < quads * CH; e += 64 * WAVES) {
            const int pos0 = (quad0 + e / CH) * 4, d = e % CH * E;
            const size_t at = ((layer_page + pages[pos0 >> 4]) * a.Hkv + g) * head;
            T *kp = static_cast<T*>(a.k_pool) + at, *vp = static_cast<T*>(a.v_pool) + at;
            union {
                u32x4 u;
                T x[E];
            } kk[4], vv[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int j = min(max(pos0 + i - L, 0), n - 1);
                kk[i].u = *reinterpret_cast<const u32x4*>(static_cast<const T*>(a.k) + (size_t)(row0 + j) * a.k_stride + g * D + d);
                vv[i].u = *reinterpret_cast<const u32x4*>(static_cast<const T*>(a.v) + (size_t)(row0 + j) * a.v_stride + g * D + d);
            }
            const bool whole = pos0 >= L && pos0 + 4 <= L + n;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int slot = (pos0 & 15) + i;
                if (pos0 + i < L || pos0 + i >= L + n) continue;
                if constexpr (F32) {
                    *reinterpret_cast<u32x4*>(kp + slot * D + d) = kk[i].u;
                    *reinterpret_cast<u32x4*>(vp + slot * D + d) = vv[i].u;
                } else {
                    *reinterpret_cast<u32x4*>(kp + kpage_offset(slot, d)) = kk[i].u;
                    if (!whole)
#pragma unroll
                        for (int x = 0; x < 8; x++) vp[vpage_offset(slot, d + x)] = vv[i].x[x];
                }
            }
            if constexpr (!F32)
                if (whole)
#pragma unroll
                    for (int x = 0; x < 8; x++)
                        *reinterpret_cast<uint2*>(vp + vpage_offset(pos0 & 15, d + x)) =
                            make_uint2((uint32_t)vv[0].x[x] | ((uint32_t)vv[1].x[x] << 16), (uint32_t)vv[2].x[x] | ((uint32_t)vv[3].x[x] << 16));
        }
    };
    const bool stores = last && r0 == 0;

    uint32_t bad[2] = {sh.bad[0], sh.bad[1]};
    if (n_items > 1) {
        // Handing over without a device-wide fence: states are stored and read with device-scope accesses, and the counter is raised only
        // when this workgroup's stores have been acknowledged.
        const size_t slot = slot0 + (size_t)(w - w0) * NR;   // of this item's first tile
        float* po = a.t.part_o + (slot + rw) * (DT * 256) + dt0 * 256 + lane;
        float* pm = a.t.part_ml + slot * 32 + rw * 16 + lr;
        if (mine) {
            if (tg == 0 && lg == 0) {
                __hip_atomic_store(pm, m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                __hip_atomic_store(pm + ROWS, lsum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
#pragma unroll
            for (int i = 0; i < OWN; i++)
#pragma unroll
                for (int e = 0; e < 4; e++) __hip_atomic_store(po + i * 256 + e * 64, own[i][e], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        uint32_t* arrive = reinterpret_cast<uint32_t*>(a.t.arrive + 4 * w0);   // counter, -, the two words of `bad`
        if (last && tid < 2) __hip_atomic_store(arrive + 2 + tid, tid ? bad[1] : bad[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (tid == 0) {
            const uint32_t old = __hip_atomic_fetch_add(arrive, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            sh.last = old == (uint32_t)n_items - 1;
            if (sh.last) __hip_atomic_store(arrive, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // for the next layer
        }
        __syncthreads();
        if (!sh.last) {
            if (stores) store_nodes();
            return;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
        bad[0] = __hip_atomic_load(arrive + 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        bad[1] = __hip_atomic_load(arrive + 3, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (mine) {
            m = NEG_BIG;
            lsum = 0.f;
#pragma unroll
            for (int i = 0; i < OWN; i++) own[i] = float4_t{0.f, 0.f, 0.f, 0.f};
            constexpr int AHEAD = 4;   // states asked for together
            for (int c0 = 0; c0 < n_items; c0 += AHEAD) {   // in ascending order, whichever came last
                float im[AHEAD], il[AHEAD], io[AHEAD][OWN][4];
#pragma unroll
                for (int c = 0; c < AHEAD; c++) {
                    const size_t from = slot0 + (size_t)min(c0 + c, n_items - 1) * stride * NR;
                    const float* qo = a.t.part_o + (from + rw) * (DT * 256) + dt0 * 256 + lane;
                    const float* qm = a.t.part_ml + from * 32 + rw * 16 + lr;
                    im[c] = __hip_atomic_load(qm, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    il[c] = __hip_atomic_load(qm + ROWS, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
                    for (int i = 0; i < OWN; i++)
#pragma unroll
                        for (int e = 0; e < 4; e++) io[c][i][e] = __hip_atomic_load(qo + i * 256 + e * 64, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
#pragma unroll
                for (int c = 0; c < AHEAD; c++) {
                    if (c0 + c >= n_items) continue;
                    const float mnew = fmaxf(m, im[c]), fo = exp2f(m - mnew), fi = exp2f(im[c] - mnew);
                    m = mnew;
                    lsum = lsum * fo + il[c] * fi;
#pragma unroll
                    for (int i = 0; i < OWN; i++)
#pragma unroll
                        for (int e = 0; e < 4; e++) own[i][e] = own[i][e] * fo + io[c][i][e] * fi;
                }
            }
        }
    }

    // the output: row lr of the tile, dims (dt0 + i) * 16 + lg * 4 ..
    if (node < n) {
        const int j = node, h = g * G + hh;
        const float inv = 1.0f / lsum;
        if (a.lse && tg == 0 && lg == 0) a.lse[(size_t)(row0 + j) * a.Hq + h] = (m + log2f(lsum)) * 0.6931471805599453f;
        const uint64_t poison = (bad[0] | bad[1]) ? seen & (((uint64_t)bad[1] << 32) | bad[0]) : 0ull;
#pragma unroll
        for (int i = 0; i < OWN; i++) {
            const int d = (dt0 + i) * 16 + lg * 4;
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; e++) y[e] = own[i][e] * inv;
            for (uint64_t left = poison; left; left &= left - 1) {   // values that are not finite, of nodes that this row sees
                const T* vp = static_cast<const T*>(a.v) + (size_t)(row0 + __builtin_ctzll(left)) * a.v_stride + g * D + d;
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (not_finite(vp[e])) {
                        if constexpr (F32) y[e] += vp[e];
                        else y[e] += bf16_to_f32(vp[e]);
                    }
            }
            if constexpr (F32) {
                *reinterpret_cast<float4*>(static_cast<float*>(a.out) + ((size_t)(row0 + j) * a.Hq + h) * D + d) = make_float4(y[0], y[1], y[2], y[3]);
            } else if constexpr (STEP) {
                bf16_t* x = static_cast<bf16_t*>(a.out) + frag_offset(row0 + j, h * D + d, a.Hq * D);
                uint32_t hi[2], lo[2];
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const bf16_t h0 = f32_to_bf16(y[2 * e]), h1 = f32_to_bf16(y[2 * e + 1]);
                    hi[e] = (uint32_t)h0 | ((uint32_t)h1 << 16);
                    lo[e] = (uint32_t)f32_to_bf16(y[2 * e] - bf16_to_f32(h0)) | ((uint32_t)f32_to_bf16(y[2 * e + 1] - bf16_to_f32(h1)) << 16);
                }
                *reinterpret_cast<uint2*>(x) = make_uint2(hi[0], hi[1]);
                *reinterpret_cast<uint2*>(x + a.x_plane) = make_uint2(lo[0], lo[1]);
            } else {
                // the conversion in hardware: to nearest even, infinities and NaN kept
                union {
                    __bf16 b[4];
                    uint2 u;
                } z;
#pragma unroll
                for (int e = 0; e < 4; e++) z.b[e] = (__bf16)y[e];
                *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.out) + ((size_t)(row0 + j) * a.Hq + h) * D + d) = z.u;
            }
        }
    }
    if (stores) store_nodes();
}

template <int D, bool F32, bool STEP>
__global__ __launch_bounds__(64 * WAVES, 2) void tree_attention_kernel(tree_args a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ tree_shared sh;
    const int32_t* rec = a.t.items + SLED_TREE_ITEM * blockIdx.x;
    switch (rec[13]) {
        case 8: attend_item<8, D, F32, STEP>(a, rec, smem, sh); break;
        case 4: attend_item<4, D, F32, STEP>(a, rec, smem, sh); break;
        default: attend_item<2, D, F32, STEP>(a, rec, smem, sh);
    }
}

// mass[token] += sum over the rows of a block and the G heads of a kv head of exp(s - lse), one more pass over K.
// S = Q K^T with the tokens on the lanes (A operand Q, B operand K), so that a lane adds up its token's weights over all rows in one
// register and nothing but the last sum crosses lanes.  A wavefront holds MP pages of K in registers and walks through
// the row tiles, whose operands all wavefronts of the workgroup share in LDS.  A token's sum is made by one
// lane group in a fixed order: no atomics, and the same result every time.
// What bounds it: 16 requests of 982 pages and 84 rows, 8 kv heads, take 16 us a layer, 7 of them K from memory, the walk 8; one request of 30011 tokens and
// 512 rows 64 us, the walk 41 of them: a tile of 16 rows against 32 tokens holds a SIMD's port for 250 clocks (8 matrix instructions of 8 clocks,
// 26 vector ones, 8 exponentials of 9) of 366 measured.  Four pages a wavefront leave room for one workgroup a CU: 18 and 79 us.
constexpr int MASS_WAVES = 8;
template <bool F32>
__host__ __device__ constexpr int mass_pages() { return 2; }   // pages of a wavefront at a time
__host__ __device__ constexpr int mass_rows(int PL) { return PL == 1 ? 256 : 128; }   // rows in LDS at a time

struct mass_args {
    float* mass;   // [request][layer][kv head][cap]
    int cap, n_layers;
};

// (two workgroups a CU where the registers allow it)
template <int D, bool F32, int PL>
__global__ __launch_bounds__(64 * MASS_WAVES, PL == 1 && !F32 ? 4 : 2) void tree_mass_kernel(tree_args a, mass_args ma) {
    constexpr int MP = mass_pages<F32>(), QT = Geo<D, F32>::QC * 64 * PL, MR = mass_rows(PL);
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int32_t* rec = a.t.mass_items + 8 * blockIdx.x;
    const int req = rec[0], g = rec[1], page0 = rec[2], npg = rec[3], n = rec[4], row0 = rec[5];
    const int32_t* pages = a.t.pages + rec[6];
    const int L = a.len_dev[req], G = a.Hq / a.Hkv, rows = G * n;
    const int page_end = min(page0 + npg, (L + n + 15) >> 4);
    if (page0 >= page_end) return;
    const int lr = lane & 15, lg = lane >> 4;
    u32x4* qs = reinterpret_cast<u32x4*>(smem);
    const int room = min(MR, (rows + 15) & ~15);
    float* lse2 = reinterpret_cast<float*>(smem + (size_t)room * PL * D * Geo<D, F32>::ELEM);   // log2 of a row's denominator
    uint64_t* seen = reinterpret_cast<uint64_t*>(lse2 + room);
    const size_t head = (size_t)16 * D, layer_page = (size_t)a.layer * a.n_pages;
    using T = std::conditional_t<F32, float, bf16_t>;
    constexpr int CHUNK = D * Geo<D, F32>::ELEM / 16 * PL, NT = 64 * MASS_WAVES, ASK = 4;
    static_assert(MR <= NT, "a thread for every row");
    for (int pb = page0; pb < page_end; pb += MASS_WAVES * MP) {
        const int p0 = pb + wave * MP;   // this wavefront's pages
        const bool stage_first = rows > MR || pb == page0;   // (rows that all fit stay where they are)
        if (pb > page0) __syncthreads();
        // Rows are asked for before they are needed: the first before the keys, so that they can be put in place while the keys are still on
        // their way, the next before the products with those in LDS.
        u32x4 x[ASK];
        float lse = 0.f;
        uint64_t sees = 0;
        auto ask = [&](int r0) __attribute__((always_inline)) {
            ask_queries<D, F32, PL>(x, a, row0, g, G, r0, rows, tid, NT);
            const int r = min(r0 + tid, rows - 1), j = r / G, h = g * G + r - j * G;
            lse = a.lse[(size_t)(row0 + j) * a.Hq + h];
            sees = a.t.seen[row0 + j];
        };
        if (stage_first) ask(0);
        Keys<D, F32> kv[MP];
        float* row = ma.mass + (((size_t)req * ma.n_layers + a.layer) * a.Hkv + g) * ma.cap;
        float had[MP], acc[MP];
#pragma unroll
        for (int p = 0; p < MP; p++) {
            const int phys = pages[min(p0 + p, page_end - 1)];
            const T* kp = static_cast<const T*>(a.k_pool) + ((layer_page + phys) * a.Hkv + g) * head;
            if constexpr (!F32) {
#pragma unroll
                for (int c = 0; c < 4; c++) kv[p].k[0][c] = reinterpret_cast<const u32x4*>(kp)[c * 64 + lane];
            } else {
#pragma unroll
                for (int c = 0; c < D / 16; c++) kv[p].k[c] = *reinterpret_cast<const f32x4*>(kp + lr * D + lg * 4 + 16 * c);
            }
            // a node's slot holds no mass of its own yet, but perhaps that of a node that was not accepted
            const int pos = (p0 + p) * 16 + lr;
            had[p] = pos < L ? row[pos] : 0.f;
            acc[p] = 0.f;
        }
        for (int r0 = 0; r0 < rows; r0 += MR) {
            const int n_rows = min(MR, (rows - r0 + 15) & ~15);
            if (r0 || stage_first) {
                if (r0) __syncthreads();
                put_queries<D, F32, PL>(qs, x, r0, n_rows, rows, tid, NT);
                for (int e0 = tid + ASK * NT; e0 < n_rows * CHUNK; e0 += ASK * NT) {
                    ask_queries<D, F32, PL>(x, a, row0, g, G, r0, rows, e0, NT);
                    put_queries<D, F32, PL>(qs, x, r0, n_rows, rows, e0, NT);
                }
                if (tid < n_rows) {
                    // a row that does not exist has an infinite denominator: its weights are zero
                    lse2[tid] = r0 + tid < rows ? lse * 1.4426950408889634f : INFINITY;
                    seen[tid] = r0 + tid < rows ? sees : 0ull;
                }
                __syncthreads();
                if (r0 + MR < rows) ask(r0 + MR);
            }
            if (p0 >= page_end) continue;
            auto walk = [&](auto masked) __attribute__((always_inline)) {
                for (int t = 0; t < n_rows / 16; t++) {
                    const float4 z = *reinterpret_cast<const float4*>(lse2 + t * 16 + lg * 4);   // of the rows this lane has
                    const float zz[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
                    for (int p = 0; p < MP; p++) {
                        const float4_t s = page_scores<D, F32, PL>(kv[p], 0, qs + t * QT + lane);
                        float sum = 0.f;
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            // (scale and denominator in log2 units are off by half a step of 2^-23 of themselves, as the score's own sum is: 3e-8 to
                            // 1.7e-7 of the masses of 14 batches together, 3e-8 to 7e-8 where lse itself is taken off.  That would be one more
                            // instruction for each of a tile's elements, which are what the kernel is bound by)
                            float e = __builtin_amdgcn_exp2f(fmaf(s[i], a.scale_log2, -zz[i]));
                            if (decltype(masked)::value) {
                                const int c = (p0 + p) * 16 + lr - L;   // node of this lane's token, if not context
                                const bool on = c < 0 || (c < n && ((seen[t * 16 + lg * 4 + i] >> (c & 63)) & 1ull));
                                e = on ? e : 0.f;
                            }
                            sum = i ? sum + e : e;
                        }
                        acc[p] += sum;
                    }
                }
            };
            if ((p0 + MP) * 16 > L) walk(std::true_type{});
            else walk(std::false_type{});
        }
        if (p0 >= page_end) continue;
#pragma unroll
        for (int p = 0; p < MP; p++) {
            const float sum = sum_over_groups(acc[p]);
            const int pos = (p0 + p) * 16 + lr;
            if (lg == 0 && p0 + p < page_end && pos < L + n) row[pos] = had[p] + sum;
        }
    }
}

// The QKV projection's K slices of row t, added up and rotated: q as a bf16 pair (fp32 models: as it is), k and v in the model's type, all as
// plain rows.  A thread takes four neighbouring rotary pairs of a q or k head or four dims of a v head.
template <bool F32>
__global__ __launch_bounds__(256) void tree_qkv_kernel(const float* __restrict__ partial, int n_split, int T_pad, int Hq, int Hkv, int D, const float2* __restrict__ cs,
                                                       void* __restrict__ Q, size_t q_plane, void* __restrict__ K, void* __restrict__ V) {
    const int t = blockIdx.x, half = D / 2, per_head = half / 4, n_rot = (Hq + Hkv) * per_head, n_qkv = (Hq + 2 * Hkv) * D;
    const int item = blockIdx.y * 256 + threadIdx.x;
    const float* row = partial + (size_t)t * n_qkv;
    const size_t slice = (size_t)T_pad * n_qkv;
    auto add = [&](int col) {
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s0 = 0; s0 < n_split; s0 += 4) {   // four slices in flight, added in ascending order
            float4 y[4];
#pragma unroll
            for (int s = 0; s < 4; s++) y[s] = s0 + s < n_split ? *reinterpret_cast<const float4*>(row + (s0 + s) * slice + col) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int s = 0; s < 4; s++) {
                x.x += y[s].x;
                x.y += y[s].y;
                x.z += y[s].z;
                x.w += y[s].w;
            }
        }
        return x;
    };
    auto pack = [](const float* y) {
        return make_uint2((uint32_t)f32_to_bf16(y[0]) | ((uint32_t)f32_to_bf16(y[1]) << 16), (uint32_t)f32_to_bf16(y[2]) | ((uint32_t)f32_to_bf16(y[3]) << 16));
    };
    auto put = [&](void* base, size_t at, const float* y) {
        if (F32) *reinterpret_cast<float4*>(static_cast<float*>(base) + at) = make_float4(y[0], y[1], y[2], y[3]);
        else *reinterpret_cast<uint2*>(static_cast<bf16_t*>(base) + at) = pack(y);
    };
    if (item < n_rot) {
        const int h = item / per_head, i = item % per_head * 4;
        const float4 c01 = *reinterpret_cast<const float4*>(cs + (size_t)t * half + i), c23 = *reinterpret_cast<const float4*>(cs + (size_t)t * half + i + 2);
        const float4 x1 = add(h * D + i), x2 = add(h * D + i + half);
        float y1[4], y2[4];
        rope_pair(x1.x, x2.x, c01.x, c01.y, y1[0], y2[0]);
        rope_pair(x1.y, x2.y, c01.z, c01.w, y1[1], y2[1]);
        rope_pair(x1.z, x2.z, c23.x, c23.y, y1[2], y2[2]);
        rope_pair(x1.w, x2.w, c23.z, c23.w, y1[3], y2[3]);
        const bool q = h < Hq;
        void* base = q ? Q : K;
        const size_t at = q ? ((size_t)t * Hq + h) * D + i : ((size_t)t * Hkv + h - Hq) * D + i;
        put(base, at, y1);
        put(base, at + half, y2);
        if (!F32 && q) {
            float l1[4], l2[4];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                l1[e] = y1[e] - bf16_to_f32(f32_to_bf16(y1[e]));
                l2[e] = y2[e] - bf16_to_f32(f32_to_bf16(y2[e]));
            }
            put(base, at + q_plane, l1);
            put(base, at + q_plane + half, l2);
        }
    } else if (item < n_rot + Hkv * (D / 4)) {
        const int e = item - n_rot;
        const float4 x = add((Hq + Hkv) * D + 4 * e);
        const float y[4] = {x.x, x.y, x.z, x.w};
        put(V, (size_t)t * Hkv * D + 4 * e, y);
    }
}

template <int D, bool F32, bool STEP>
int launch_attention(const tree_args& a, hipStream_t st) {
    constexpr size_t lds = std::max(attention_lds<2, D, F32>(), std::max(attention_lds<4, D, F32>(), attention_lds<8, D, F32>()));
    static_assert(lds + sizeof(tree_shared) <= 160 * 1024, "LDS of a workgroup");
    static bool allowed = false;
    if (!allowed) {
        SLED_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(tree_attention_kernel<D, F32, STEP>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        allowed = true;
    }
    hipLaunchKernelGGL((tree_attention_kernel<D, F32, STEP>), dim3(a.t.n_items), dim3(64 * WAVES), lds, st, a);
    SLED_LAUNCH_CHECK();
    return SLED_OK;
}

template <int D, bool F32, int PL>
int launch_mass(const tree_args& a, const mass_args& ma, int max_rows, hipStream_t st) {
    const int room = std::min(mass_rows(PL), (max_rows + 15) & ~15);
    const size_t lds = (size_t)room * (PL * D * Geo<D, F32>::ELEM + sizeof(float) + sizeof(uint64_t));
    static size_t allowed = 0;
    if (lds > allowed) {
        SLED_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(tree_mass_kernel<D, F32, PL>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        allowed = lds;
    }
    hipLaunchKernelGGL((tree_mass_kernel<D, F32, PL>), dim3(a.t.n_mass_items), dim3(64 * MASS_WAVES), lds, st, a, ma);
    SLED_LAUNCH_CHECK();
    return SLED_OK;
}

tree_args common_args(const sled_model* m, const sled_kvpool* p, const sled_tree_plan& t, int layer, const void* q, size_t q_stride, size_t q_plane) {
    tree_args a{};
    a.t = t;
    a.len_dev = p->len_dev;
    a.q = q;
    a.q_stride = q_stride;
    a.q_plane = q_plane;
    a.k_pool = p->k_pool;
    a.v_pool = p->v_pool;
    a.n_pages = p->n_pages;
    a.layer = layer;
    a.Hq = m->s.n_q_heads;
    a.Hkv = m->s.n_kv_heads;
    a.scale_log2 = 1.4426950408889634f / sqrtf((float)m->s.head_dim);
    return a;
}

}  // namespace

int sled_launch_tree_attention(const sled_model* m, const sled_kvpool* p, const sled_tree_plan& t, int layer, const void* q, size_t q_stride, size_t q_plane,
                               const void* k, size_t k_stride, const void* v, size_t v_stride, void* out, size_t x_plane, float* lse, bool step, hipStream_t st) {
    tree_args a = common_args(m, p, t, layer, q, q_stride, q_plane);
    a.k = k;
    a.v = v;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.out = out;
    a.x_plane = x_plane;
    a.lse = lse;
    if (m->s.dtype == SLED_BF16) return step ? launch_attention<128, false, true>(a, st) : launch_attention<128, false, false>(a, st);
    return m->s.head_dim == 64 ? launch_attention<64, true, false>(a, st) : launch_attention<128, true, false>(a, st);
}

int sled_launch_tree_mass(const sled_model* m, const sled_kvpool* p, const sled_tree_plan& t, int layer, const void* q, size_t q_stride, size_t q_plane,
                          const float* lse, float* mass, int cap, hipStream_t st) {
    tree_args a = common_args(m, p, t, layer, q, q_stride, q_plane);
    a.lse = const_cast<float*>(lse);
    const mass_args ma{mass, cap, m->s.n_layers};
    const int rows = t.max_nodes * (m->s.n_q_heads / m->s.n_kv_heads);
    if (m->s.dtype == SLED_BF16) return q_plane ? launch_mass<128, false, 2>(a, ma, rows, st) : launch_mass<128, false, 1>(a, ma, rows, st);
    return m->s.head_dim == 64 ? launch_mass<64, true, 1>(a, ma, rows, st) : launch_mass<128, true, 1>(a, ma, rows, st);
}

int sled_launch_tree_qkv(const sled_model* m, int T, const float* partial, int n_split, int T_pad, const float* cs, void* Q, size_t q_plane, void* K, void* V,
                         hipStream_t st) {
    const int Hq = m->s.n_q_heads, Hkv = m->s.n_kv_heads, D = m->s.head_dim;
    const dim3 grid(T, ((Hq + Hkv) * (D / 8) + Hkv * (D / 4) + 255) / 256);
    if (m->s.dtype == SLED_BF16)
        hipLaunchKernelGGL(tree_qkv_kernel<false>, grid, dim3(256), 0, st, partial, n_split, T_pad, Hq, Hkv, D, reinterpret_cast<const float2*>(cs), Q, q_plane, K, V);
    else
        hipLaunchKernelGGL(tree_qkv_kernel<true>, grid, dim3(256), 0, st, partial, n_split, T_pad, Hq, Hkv, D, reinterpret_cast<const float2*>(cs), Q, q_plane, K, V);
    SLED_LAUNCH_CHECK();
    return SLED_OK;
}
