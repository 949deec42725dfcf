// retention_common.hpp -- shared pieces of the retention kernels (linear
// attention whose state decays at a rate of its own in each head): operands of
// the bf16 matrix cores, LDS tiles of a chunk, register layouts, decay powers.
//
// One walk serves the operator and its whole gradient.  With rows i of a tape in
// walking order, W(x, y, z) is
//     state_i = gamma state_{i-1} + y_i^T z_i   (the carried part dropped at a begin)
//     W_i     = x_i state_i
// and   out = W(q, k, v),  dq = W(dout, v, k)  forwards,
//       dv  = W(k, q, dout),  dk = W(v, dout, q)  backwards in time,
// where a step "begins" backwards when the step after it begins an episode.
//
// A workgroup of VD / 16 wavefronts walks a run of chunks of C rows of one head
// with the state (KD x VD) in registers, 16 of its columns per wavefront.
//
// Every product runs on v_mfma_f32_16x16x32_bf16.  bf16 inputs go in as they
// are.  A float goes in as three bf16 planes, x = h + m + l with h and m its
// leading bits cut off: exact, 8 bits each.  Two such numbers take the six
// products of planes whose indices add to at most 2; what is left out is below
// 2^-21 of the product, which sums of 64 and more floats do not keep either: six
// bf16 instructions, 16 / 6 of the rate of the fp32 matrix cores.
//
// With lane = 16 g + c the instruction takes A[i = c][k = 8 g + e] and
// B[k = 8 g + e][j = c] and returns D[i = 4 g + r][j = c] in register r.  The
// order of the k slots is free as long as A and B share it, and so is which
// column stands in which row of A; the layouts use both so that results are
// operands of the next product where they are:
//   * rows of a chunk as k: slot (g, e) is row 32 tb + 16 (e / 4) + 4 g + e % 4.
//     The masked products P^T, two 16-row tiles, come out in that order; columns
//     of a row-major LDS tile are read in it by ds_read_b64_tr_b16;
//   * state rows kd as k: slot (g, e) is kd = 32 s + 8 g + e, as 16 bytes of a row
//     of x are.  The state tile (s, u) holds kd = 32 s + 8 (i / 4) + 4 u + i % 4 in
//     its row i, so registers of tiles (s, 0) and (s, 1) are those eight slots;
//   * a wavefront has 16 of the state's columns, and a row of the result has four
//     consecutive ones in each lane.
#pragma once

#include "scan_common.hpp"
#include "kernels.hpp"

namespace memoroid {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// NP planes per input element: 1 = bf16, 3 = float.  Chunks of float are half as
// long: the planes of three 64-row chunks of 128 columns do not fit in LDS.
template <int NP_, int KD_, int VD_>
struct RetCfg {
    static constexpr int NP = NP_, KD = KD_, VD = VD_;
    static constexpr int FP = NP == 1 ? 2 : 3;        // planes of a float as an operand (pairs' weights, the state)
    static constexpr int C = ret_chunk(NP);
    static constexpr int CW = VD / 16, W = CW, THREADS = 64 * W;   // wavefronts per state's columns, in all
    static constexpr int ES = NP == 1 ? 2 : 4;        // bytes of an element in memory
    static constexpr int EPU = 16 / ES;               // elements of a 16-byte unit
    static constexpr int NB = C / 16;                 // 16-row blocks
    static constexpr int NTILE = NB * (NB + 1) / 2;   // tiles of P on and below the diagonal
    static constexpr int KS = KD / 32;                // steps of a product over kd
};

// The same for a workgroup that holds several states: 64 of a state's rows per
// wavefront, (KD / 64) (VD / 16) wavefronts, so that four states fit.  (No product
// over the state's rows is taken there, so nothing is added up across wavefronts.)
template <class Cfg>
struct RetCfg64 : Cfg {
    static constexpr int W = Cfg::CW * (Cfg::KD / 64), THREADS = 64 * W, KS = 2;
};

struct RetLane {
    int tid, lane, w, g, c;
    int k0 = 0;                                       // first state row of the wavefront
    __device__ RetLane() {
        tid = threadIdx.x;
        w = __builtin_amdgcn_readfirstlane(tid >> 6);
        again();
    }
    // The same again, opaque to the compiler: what it derives from these is
    // recomputed in each chunk instead of being kept over the loop (a hundred
    // addresses and masks, which took the registers that the state needs).
    __device__ __forceinline__ void again() {
        asm volatile("" : "+v"(tid));
        lane = tid & 63;
        g = lane >> 4;
        c = lane & 15;
    }
};

// ------------------------------------------------------------------ planes
// the upper halves of a and b in one word, a's in the low half
__device__ __forceinline__ uint32_t pack_hi(float a, float b) {
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ float cut(float x) { return __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }
// Two floats as NPL planes of packed bf16 words.  One plane: rounded to nearest.
// Two: the rounding error rounded once more, right to 2^-17.  Three: cut, exact (an
// infinity leaves NaN in its lower planes: the products are then NaN, not infinite).
template <int NPL>
__device__ __forceinline__ void planes2(float a, float b, uint32_t (&w)[NPL]) {
    if constexpr (NPL < 3) {
        w[0] = f32x2_to_bf16x2(a, b);
        if constexpr (NPL == 2) w[1] = f32x2_to_bf16x2(a - __uint_as_float(w[0] << 16), b - cut(__uint_as_float(w[0])));
    } else {
        w[0] = pack_hi(a, b);
        a -= cut(a);
        b -= cut(b);
        w[1] = pack_hi(a, b);
        a -= cut(a);
        b -= cut(b);
        w[2] = pack_hi(a, b);
    }
}
// eight floats as operands
template <int NPL>
__device__ __forceinline__ void planes8(f32x4 lo, f32x4 hi, bf16x8 (&f)[NPL]) {
    u32x4 w[NPL];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        uint32_t x[NPL];
        if (p < 2) planes2<NPL>(lo[2 * p], lo[2 * p + 1], x);
        else planes2<NPL>(hi[2 * p - 4], hi[2 * p - 3], x);
#pragma unroll
        for (int i = 0; i < NPL; ++i) w[i][p] = x[i];
    }
#pragma unroll
    for (int i = 0; i < NPL; ++i) f[i] = __builtin_bit_cast(bf16x8, w[i]);
}
// the float that NP planes of element e stand for
template <int NP>
__device__ __forceinline__ float plane_value(const bf16x8 (&f)[NP], int e) {
    auto one = [&](int i) {
        const u32x4 w = __builtin_bit_cast(u32x4, f[i]);
        return e & 1 ? __uint_as_float(w[e >> 1] & 0xFFFF0000u) : __uint_as_float(w[e >> 1] << 16);
    };
    if constexpr (NP == 1) return one(0);
    else return one(0) + (one(1) + one(2));
}

template <int NA, int NB>
__device__ __forceinline__ void mma(f32x4& acc, const bf16x8 (&a)[NA], const bf16x8 (&b)[NB]) {
#pragma unroll
    for (int i = NA - 1; i >= 0; --i)
#pragma unroll
        for (int j = NB - 1; j >= 0; --j)
            if (i + j < 3) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[j], acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 zero4() { return f32x4{0.0f, 0.0f, 0.0f, 0.0f}; }

// --------------------------------------------------------- chunks in memory
// n rows of one head of a [T][heads][d] tensor as a buffer, from step t0 on; walking
// backwards row i is the (n - 1 - i)-th of them.  Rows at or past n lie outside the
// buffer (backwards: below offset 0, which wraps past its end), columns at or past d
// are sent there: they read as zeros and drop their stores.
struct RetRows {
    Rsrc r;
    int first, step, d;         // byte offsets of row 0 and from row to row
    __device__ __forceinline__ uint32_t offset(int row, int col, int es) const {
        return col < d ? (uint32_t)(first + row * step + col * es) : kOob;
    }
};
__device__ __forceinline__ RetRows ret_rows(const void* head0, int64_t row_bytes, int d, int es, int t0, int n, bool rev) {
    const int rb = (int)row_bytes, end = (n - 1) * rb;
    return RetRows{make_rsrc((const char*)head0 + t0 * row_bytes, n > 0 ? (int64_t)end + d * es : 0), rev ? end : 0,
                   rev ? -rb : rb, d};
}

// Where the 16-byte unit `unit` of row `row` of an LDS tile of D columns lies: the
// units of a row are exchanged by its number, so that operands take the cycles of
// their bytes and rows need no padding.  A row operand reads one unit of 16 rows,
// which lie in different banks (28 cycles more without the exchange); a column
// operand reads half a unit each of four units, a quarter of the row, in four
// neighbouring rows, so it is those rows' numbers that tell the quarters apart
// (with the quarters told apart by row / 4 they were 5.5 cycles more a read).
// Counted (128 x 128, bf16): SQ_LDS_IDX_ACTIVE of a walk is 546 cycles per wavefront
// and chunk, which moves 71 KB, 554 cycles at 128 bytes each; SQ_LDS_BANK_CONFLICT
// calls 200 of them conflicts, two of the four of every transposed read among them.
template <int D>
__device__ __forceinline__ int swizzled(int unit, int row) {
    static_assert(D == 64 || D == 128, "8 or 16 units a row");
    const int q = (row >> 2) & 3;
    return D == 128 ? unit ^ (((row & 3) << 2) | q) : unit ^ (((row & 2) << 1) | q);
}

// A chunk's tile of D columns held by the workgroup, 16 bytes a unit: thread
// `tid` has the same columns of rows tid / UPR + i RS
template <class Cfg, int D>
struct RetTile {
    static constexpr int UPR = D / Cfg::EPU, RS = Cfg::THREADS / UPR, UN = Cfg::C / RS;
    static_assert(UN >= 1 && UN * RS == Cfg::C, "every thread holds a unit");
    u32x4 u[UN];

    __device__ __forceinline__ void fetch(const RetRows& x, const RetLane& L) {
        const int col = L.tid % UPR * Cfg::EPU;
        uint32_t off = x.offset(L.tid / UPR, col, Cfg::ES);
        const uint32_t step = col < x.d ? (uint32_t)(RS * x.step) : 0u;
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            u[i] = __builtin_amdgcn_raw_buffer_load_b128(x.r, (int)off, 0, 0);
            off += step;
        }
    }
    // nonzero if some element is not finite
    __device__ __forceinline__ uint32_t bad() const {
        constexpr uint32_t kExp = Cfg::NP == 1 ? 0x7F807F80u : 0x7F800000u, kOne = Cfg::NP == 1 ? 0x00800080u : 0x00800000u;
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < UN; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) any |= (u[i][e] & kExp) + kOne;
        return any & (Cfg::NP == 1 ? 0x80008000u : 0x80000000u);
    }
    // rows from .. to - 1 stay, the others become zeros
    __device__ __forceinline__ void keep(int from, int to, const RetLane& L) {
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            const int row = L.tid / UPR + i * RS;
            if (row < from || row >= to) u[i] = u32x4{0u, 0u, 0u, 0u};
        }
    }
    // into an LDS tile of NP planes
    __device__ __forceinline__ void stage(uint16_t* s, const RetLane& L) const {
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            const int row = L.tid / UPR + i * RS, col = L.tid % UPR * Cfg::EPU;
            const u32x4 x = u[i];
            uint16_t* const p = s + row * D + swizzled<D>(col / 8, row) * 8 + col % 8;
            if constexpr (Cfg::NP == 1) {
                *(u32x4*)p = x;
            } else {
                uint32_t lo[3], hi[3];
                planes2<3>(__uint_as_float(x[0]), __uint_as_float(x[1]), lo);
                planes2<3>(__uint_as_float(x[2]), __uint_as_float(x[3]), hi);
#pragma unroll
                for (int q = 0; q < 3; ++q) *(u32x2*)(p + q * Cfg::C * D) = u32x2{lo[q], hi[q]};
            }
        }
    }
};

// ------------------------------------------------------------ LDS operands
// columns k0 + 32 s + 8 g .. + 7 of one row as floats, the same in the 16 lanes of g
template <class Cfg, int D>
__device__ __forceinline__ void row_values(float (&v)[8], const uint16_t* t, int row, int s, const RetLane& L) {
    bf16x8 f[Cfg::NP];
#pragma unroll
    for (int p = 0; p < Cfg::NP; ++p)
        f[p] = *(const bf16x8*)(t + p * Cfg::C * D + row * D + swizzled<D>(L.k0 / 8 + 4 * s + L.g, row) * 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = plane_value<Cfg::NP>(f, e);
}
// one element
template <class Cfg, int D>
__device__ __forceinline__ float tile_value(const uint16_t* t, int row, int col) {
    const uint16_t* const at = t + row * D + swizzled<D>(col >> 3, row) * 8 + (col & 7);
    const float h = __uint_as_float((uint32_t)at[0] << 16);
    if constexpr (Cfg::NP == 1) return h;
    else return h + (__uint_as_float((uint32_t)at[Cfg::C * D] << 16) + __uint_as_float((uint32_t)at[2 * Cfg::C * D] << 16));
}
// 16 rows from row0 (a multiple of 16), columns 32 s + 8 g ..: a row operand
template <class Cfg, int D>
__device__ __forceinline__ void row_frag(bf16x8 (&f)[Cfg::NP], const uint16_t* t, int row0, int s, const RetLane& L) {
#pragma unroll
    for (int p = 0; p < Cfg::NP; ++p)
        f[p] = *(const bf16x8*)(t + p * Cfg::C * D + (row0 + L.c) * D + swizzled<D>(4 * s + L.g, L.c) * 8);
}
// rows 32 tb .. + 31 as k, the column of `col` (of this lane's address: four
// consecutive columns from there): a column operand
template <class Cfg, int D>
__device__ __forceinline__ void col_frag(bf16x8 (&f)[Cfg::NP], const uint16_t* t, int tb, int col, const RetLane& L) {
    typedef __attribute__((address_space(3))) s16x4* LdsPtr;
    const int row = 4 * L.g + (L.c >> 2);                  // of 16
    const uint16_t* const t0 = t + (32 * tb + row) * D + swizzled<D>(col >> 3, row) * 8 + (col & 7);
#pragma unroll
    for (int p = 0; p < Cfg::NP; ++p) {
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(t0 + p * Cfg::C * D));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(t0 + p * Cfg::C * D + 16 * D));
        f[p] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
}

// ---------------------------------------------------------------- the state
// S[s][u], rows as above.  The column and the rows of this lane, and those of its
// address in col_frag (four columns from there)
template <class Cfg>
using State = f32x4[Cfg::KS][2];

__device__ __forceinline__ int state_col(const RetLane& L) { return 16 * L.w + L.c; }
__device__ __forceinline__ int state_col_addr(const RetLane& L) { return 16 * L.w + 4 * (L.c & 3); }
__device__ __forceinline__ int state_row(int s, int u, int r, const RetLane& L) {
    return L.k0 + 32 * s + 8 * L.g + 4 * u + r;
}
__device__ __forceinline__ int state_row_addr(int s, int u, const RetLane& L) {
    return L.k0 + 32 * s + 8 * (L.c & 3) + 4 * u;
}

template <class Cfg, class F>
__device__ __forceinline__ void each(State<Cfg>& S, F&& f) {
#pragma unroll
    for (int s = 0; s < Cfg::KS; ++s)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) S[s][u][e] = f(S[s][u][e], s, u, e);
}
template <class Cfg>
__device__ __forceinline__ void zero_state(State<Cfg>& S) {
    each<Cfg>(S, [](float, int, int, int) { return 0.0f; });
}
// An array of kd x vd floats with strides sk, sv: zeros where there is none
template <class Cfg>
__device__ __forceinline__ void load_state(State<Cfg>& S, const float* p, int sk, int sv, int kd, int vd,
                                           const RetLane& L) {
    const Rsrc r = make_rsrc(p, p ? (int64_t)kd * vd * 4 : 0);
    const int v = state_col(L);
    each<Cfg>(S, [&](float, int s, int u, int e) {
        const int k = state_row(s, u, e, L);
        const uint32_t off = k < kd && v < vd ? (uint32_t)(k * sk + v * sv) * 4u : kOob;
        return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, (int)off, 0, 0));
    });
}
template <class Cfg>
__device__ __forceinline__ void store_state(State<Cfg>& S, float* p, int sk, int sv, int kd, int vd, float mul, bool drop,
                                            const RetLane& L) {
    const Rsrc r = make_rsrc(p, (int64_t)kd * vd * 4);
    const int v = state_col(L);
    each<Cfg>(S, [&](float x, int s, int u, int e) {
        const int k = state_row(s, u, e, L);
        const uint32_t off = k < kd && v < vd ? (uint32_t)(k * sk + v * sv) * 4u : kOob;
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(drop ? 0.0f : x * mul), r, (int)off, 0, 0);
        return x;
    });
}

// ------------------------------------------------------------------- decays
// gamma^n = exp(-rate n), formed in 64 bits: a slow rate compounds over 1e5
// steps, where the rounding of a 32-bit gamma^C would show.
__device__ __forceinline__ float decay_pow(double rate, double n) { return n == 0.0 ? 1.0f : (float)exp(-rate * n); }
// a value that is the same in all lanes, kept once
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float uniform(float x) { return __uint_as_float((uint32_t)uniform((int)__float_as_uint(x))); }
__device__ __forceinline__ double uniform(double x) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, (uint64_t)(uint32_t)uniform((int)(uint32_t)b) |
                                          (uint64_t)(uint32_t)uniform((int)(uint32_t)(b >> 32)) << 32);
}
// x -> gamma^n x with gamma^n = hi + lo to 48 bits: a rounded factor near 1 would
// be off the same way every time (16384 steps at a rate of 1/4096: 1.1e-4 of the
// state, 2.5e-7 so).  The large product is the one that the fma leaves unrounded:
// rounded first, it would lose what lo adds.
struct Carry {
    float hi, lo;
    __device__ __forceinline__ float operator()(float x) const { return __builtin_fmaf(x, hi, x * lo); }
};
__device__ __forceinline__ Carry carry_by(double p) {
    return Carry{uniform((float)p), uniform((float)(p - (double)(float)p))};
}
__device__ __forceinline__ Carry carry_of(double rate, double n) { return carry_by(n == 0.0 ? 1.0 : exp(-rate * n)); }
template <class Cfg>
__device__ __forceinline__ void carry_state(State<Cfg>& S, Carry cy) {
    each<Cfg>(S, [&](float x, int, int, int) { return cy(x); });
}

// The decay of a walk's state that its registers have not taken yet: state =
// now S, with what is added divided by `now`.  They take it when it passes 2^-20,
// which keeps the quotients far from float's range; a slow head almost never
// does, and none pays 64 instructions a chunk for it.  All in 64 bits.  (A rate
// that is NaN makes them take it too.)
struct Owed {
    double now = 1.0, inverse = 1.0;
    __device__ __forceinline__ void none() { now = inverse = 1.0; }
    // n steps of decay more; whether the registers have to take `now`
    template <class Powers>
    __device__ __forceinline__ bool add(const Powers& p, int n) {
        now = uniform(now * p.of[n]);
        inverse = uniform(inverse * p.inverse[n]);
        return !(now >= 0x1p-20);
    }
};
// gamma^n and its inverse for n = 0 .. N - 1, in LDS
template <int N>
struct Powers {
    double of[N], inverse[N];
    __device__ __forceinline__ void fill(double rate, int tid) {
        if (tid < N) {
            of[tid] = tid == 0 ? 1.0 : exp(-rate * tid);
            inverse[tid] = tid == 0 ? 1.0 : exp(rate * tid);
        }
    }
    __device__ __forceinline__ float f(int n) const { return (float)of[n]; }
};

// What a chunk makes of the state before it: nothing is left where a step begins,
// else it takes the decay it owes if it has to.  The asm keeps the state in one
// set of registers; the ways through the branches got one each, and spilled.
template <class Cfg>
__device__ __forceinline__ void settle(State<Cfg>& S, bool begins, bool take, Carry cy) {
    if (begins) zero_state<Cfg>(S);
    each<Cfg>(S, [&](float x, int, int, int) {
        asm volatile("" : "+v"(x));
        return x;
    });
    if (take) carry_state<Cfg>(S, cy);
    each<Cfg>(S, [&](float x, int, int, int) {
        asm volatile("" : "+v"(x));
        return x;
    });
}

// ----------------------------------------------------------------- begins
// The begin flag of row `lane` of a chunk of n steps from t0 on, 0 past them:
// backwards row i is step t0 + n - 1 - i and begins if the step after it does (the
// last step of the tape goes on from what follows it).
__device__ __forceinline__ uint32_t ret_flag(const uint8_t* start, int t0, int n, int T, bool rev, int lane) {
    const int low = rev ? t0 + 1 : t0, left = T - low;     // the lowest step looked at
    const Rsrc r = make_rsrc(start + low, n <= 0 ? 0 : left < n ? left : n);
    return bload_u8(r, (uint32_t)(rev ? n - 1 - lane : lane));
}
__device__ __forceinline__ uint64_t upto(int i) { return (2ull << i) - 1ull; }          // bits 0 .. i
__device__ __forceinline__ int last_begin(uint64_t m) { return 63 - __builtin_clzll(m); }   // m != 0

}  // namespace memoroid
