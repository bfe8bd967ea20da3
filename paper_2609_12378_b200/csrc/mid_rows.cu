// What lies between the two column-wise kernels of a key switch whose digits serve one key: the forward row pass of the extended
// digits, their inner product with the key, and the inverse row pass of the limbs that ModDown converts.
//
// sigma_g maps rows of 256 words onto rows (a word's row is the low part of its bit-reversed index, and the low part of g (2 b + 1)
// follows from the low part of b), so that a row of the result needs one row of each digit: nothing but the sums leaves the SM,
// where the digits' evaluation form made a trip through memory (36 MiB out and 96 MiB in per ciphertext at N = 2^16, level 24) and
// two launches were one more.  Digits that many keys share (hoisted rotations, baby steps) keep that form: it is computed once.
#include "butterfly.cuh"

namespace {

// A warp per row, eight coefficients per lane (stages in groups of 3, 3 and 2), so that the sums of both components fit 64 registers:
// the kernel waits for its key words and digits, and 32 warps per SM wait for more of them at a time (16 lanes per row with
// sixteen coefficients and 128 registers: 54 us for one ciphertext at N = 2^16, level 24).  Sums over terms hold theirs throughout, and at
// five CTAs per SM those of three and four digits spill (144 and 220 bytes per thread stored).
constexpr uint32_t MID_ROWS = 4;

template <uint32_t BETA, bool TERMS>
__global__ void __launch_bounds__(32 * MID_ROWS, TERMS ? 5 : 8) mid_rows(DevTables c, const __grid_constant__ MidArgs a) {
    __shared__ __align__(16) double sm[BETA][MID_ROWS][WROW_PAD];
    const uint32_t t = threadIdx.x & 31, rl = threadIdx.x >> 5, row = blockIdx.x * MID_ROWS + rl, R = c.N >> 8;
    // special limbs, which have the most to do, first: they would stretch the last wave (rotation at N = 2^15 42.6 -> 40.8 us, at
    // N = 2^16 150.9 -> 149.7)
    const uint32_t bz = blockIdx.y, nt = a.level + c.K, x = TERMS ? blockIdx.z : nt - 1 - blockIdx.z, kt = x < a.level ? x : c.L + (x - a.level);
    const double q = c.modd[kt].x, qinv = c.modd[kt].y;
    const uint32_t p0 = row * 256 + 2 * t, own = x < a.level ? x / c.alpha : BETA;       // own: the digit that has x among its own limbs
    const size_t limb = (size_t)1 << c.log_n;
    double s0[8], s1[8];               // sums of words p0 + 64 k, p0 + 64 k + 1 of both components
    if (TERMS)
#pragma unroll
        for (uint32_t k = 0; k < 8; k++) s0[k] = s1[k] = 0.0;
    grid_dep_sync();
    const uint32_t nterm = TERMS ? a.nterm : 1;
#pragma unroll 1
    for (uint32_t term = 0; term < nterm; term++) {
        const uint32_t key = a.group ? bz / a.group : term;
        const uint32_t gal = (uint32_t)a.galois[key], srow = galois_src(row << 8, gal, c.log_n) >> 8;
#pragma unroll 1
        for (uint32_t j = 0; j < BETA; j++) {
            double *s = sm[j][rl];
            if (j == own) {
                const u64 *d = a.d.at(term * a.nb + bz) + x * limb + srow * 256 + 2 * t;
                ulonglong2 w[4];
#pragma unroll
                for (uint32_t k = 0; k < 4; k++) w[k] = ld_pair<true>(d + 64 * k);
#pragma unroll
                for (uint32_t k = 0; k < 4; k++) *reinterpret_cast<double2 *>(s + wrow_at(2 * t) + 72 * k) = make_double2(u64_to_d(w[k].x), u64_to_d(w[k].y));
                continue;
            }
            const double *tw = c.twd_fwd + ((size_t)kt << c.log_n);
            const double *g = reinterpret_cast<const double *>(a.ext + term * a.term_stride) + (((size_t)bz * BETA + j) * nt + x) * limb + srow * 256 + t;
            double v[8];
#pragma unroll
            for (uint32_t k = 0; k < 8; k++) v[k] = g[32 * k];
            wrow_forward(v, s, t, tw, R + srow, q, qinv);
        }
        __syncwarp();
        const u64 *c0 = TERMS && x < a.level && a.c0[term] ? a.c0[term] + bz * a.c0_stride + x * limb + srow * 256 : nullptr;
        const u64 *kp = a.evk[key] + kt * limb + p0;
        const size_t kc = c.T * limb;          // from a key's component to the next, digit by digit
#pragma unroll
        for (uint32_t k = 0; k < 4; k++) {
            const uint32_t sr = galois_src(p0 + 64 * k, gal, c.log_n) & 255, so = sr & ~1u;
            const bool odd = sr & 1;             // the permutation maps the pair onto a pair, possibly swapped
            ulonglong2 kv[BETA][2];
#pragma unroll
            for (uint32_t j = 0; j < BETA; j++) {
                kv[j][0] = ld_pair<true>(kp + 2 * j * kc + 64 * k);
                kv[j][1] = ld_pair<true>(kp + (2 * j + 1) * kc + 64 * k);
            }
            if (!TERMS) s0[2 * k] = s0[2 * k + 1] = s1[2 * k] = s1[2 * k + 1] = 0.0;
            if (TERMS && c0) {
                const ulonglong2 z = ld_pair<true>(c0 + so);
                const double pq = c.dn_p_mod_d[x];
                s0[2 * k] = __dadd_rn(s0[2 * k], mulmod_dd(u64_to_d(odd ? z.y : z.x), pq, q, qinv));
                s0[2 * k + 1] = __dadd_rn(s0[2 * k + 1], mulmod_dd(u64_to_d(odd ? z.x : z.y), pq, q, qinv));
            }
#pragma unroll
            for (uint32_t j = 0; j < BETA; j++) {
                const double2 e = *reinterpret_cast<const double2 *>(sm[j][rl] + wrow_at(so));
                const double e0 = odd ? e.y : e.x, e1 = odd ? e.x : e.y;
                s0[2 * k] = __dadd_rn(s0[2 * k], mulmod_dd(e0, u64_to_d(kv[j][0].x), q, qinv));
                s0[2 * k + 1] = __dadd_rn(s0[2 * k + 1], mulmod_dd(e1, u64_to_d(kv[j][0].y), q, qinv));
                s1[2 * k] = __dadd_rn(s1[2 * k], mulmod_dd(e0, u64_to_d(kv[j][1].x), q, qinv));
                s1[2 * k + 1] = __dadd_rn(s1[2 * k + 1], mulmod_dd(e1, u64_to_d(kv[j][1].y), q, qinv));
            }
            // at most BETA + 1 products of 0.75 q on top of half a prime
            s0[2 * k] = reduce_d(s0[2 * k], q, qinv); s0[2 * k + 1] = reduce_d(s0[2 * k + 1], q, qinv);
            s1[2 * k] = reduce_d(s1[2 * k], q, qinv); s1[2 * k + 1] = reduce_d(s1[2 * k + 1], q, qinv);
            asm volatile("" ::: "memory");       // one step's words at a time: the registers hold no more
        }
        __syncwarp();
    }
    // what is added in place: P times a ciphertext (q-limbs), or the sum that u holds
    const u64 *add = a.has_add && x < a.level ? a.add.at(bz) + x * limb + p0 : nullptr;
    u64 *u = a.u + ((size_t)bz * 2 * nt + x) * limb + p0;
    const double *twi = c.twd_inv + ((size_t)kt << c.log_n);
#pragma unroll
    for (uint32_t cm = 0; cm < 2; cm++, u += nt * limb) {
        double (&v)[8] = cm ? s1 : s0;
        if (add || a.acc_u) {
            const u64 *o = add ? add + cm * a.level * limb : u;
            const double pq = add ? c.dn_p_mod_d[x] : 1.0;
#pragma unroll
            for (uint32_t k = 0; k < 4; k++) {
                const ulonglong2 z = ld_pair<true>(o + 64 * k);
                v[2 * k] = reduce_d(__dadd_rn(v[2 * k], mulmod_dd(u64_to_d(z.x), pq, q, qinv)), q, qinv);
                v[2 * k + 1] = reduce_d(__dadd_rn(v[2 * k + 1], mulmod_dd(u64_to_d(z.y), pq, q, qinv)), q, qinv);
            }
        }
        if (x < a.inv_from) {
#pragma unroll
            for (uint32_t k = 0; k < 4; k++) st_pair<true>(u + 64 * k, make_ulonglong2(canonical_d(v[2 * k], q), canonical_d(v[2 * k + 1], q)));
            continue;
        }
        double *s = sm[0][rl];
#pragma unroll
        for (uint32_t k = 0; k < 4; k++) *reinterpret_cast<double2 *>(s + wrow_at(2 * t) + 72 * k) = make_double2(v[2 * k], v[2 * k + 1]);
        __syncwarp();
        wrow_inverse(v, s, t, twi, R + row, q, qinv);
        double *g = reinterpret_cast<double *>(u) - t;
#pragma unroll
        for (uint32_t k = 0; k < 8; k++) g[32 * k] = v[k];
        __syncwarp();
    }
}

// The same for rotations whose results are multiplied by plaintexts (PosArgs): every rotation reads the one set of digits through its own
// permutation, its sums meet their factor S_r in registers, and the ciphertext's own term comes on top.  Products are summed exactly and reduced
// once (ProductSum).  Bound by two pipes at a time, FP64 65 % and the load/store unit's shared-memory and L1 passes 69 % of their cycles (sixteen
// ciphertexts at N = 2^16, level 24: 563 us; 656 with every product reduced and the sums of a row kept until its end).  Warps of a CTA take the
// same row of up to four ciphertexts, which share its key words, twiddles and often plaintexts in L1 (L2 hits instead: 3 % more).  Tried and
// slower or no faster there: the words on their way to L2 ahead of the digits' transforms (629 us then, no change), the row's twiddles in
// shared memory (no change), one component after the other (632), eight CTAs per SM at 64 registers (578, spilling).
struct PosRow {            // a warp's place
    uint32_t t, rl, row, R, bz, nt, x, kt, own, set;
    double q, qinv, pq;
    size_t limb, cc, kc;
};
__device__ __forceinline__ PosRow pos_row(const DevTables &c, const PosArgs &a, uint32_t beta, uint32_t row, uint32_t bz) {
    PosRow p;
    p.t = threadIdx.x & 31; p.rl = threadIdx.x >> 5; p.R = c.N >> 8;
    p.row = row; p.bz = bz;
    p.nt = a.level + c.K;
    p.x = p.nt - 1 - blockIdx.z; p.kt = p.x < a.level ? p.x : c.L + (p.x - a.level);
    p.own = p.x < a.level ? p.x / c.alpha : beta;           // the digit that has x among its own limbs
    p.set = a.set[p.bz & (KS_MULTI - 1)];
    p.q = c.modd[p.kt].x; p.qinv = c.modd[p.kt].y;
    p.pq = p.x < a.level ? c.dn_p_mod_d[p.x] : 0.0;
    p.limb = (size_t)1 << c.log_n; p.cc = a.pitch * p.limb; p.kc = c.T * p.limb;
    return p;
}
// a CTA's warps as MID_ROWS / 2^share rows of 2^share entries
__device__ __forceinline__ PosRow pos_warp(const DevTables &c, const PosArgs &a, uint32_t beta) {
    const uint32_t w = threadIdx.x >> 5;
    return pos_row(c, a, beta, blockIdx.x * (MID_ROWS >> a.share) + (w >> a.share), (blockIdx.y << a.share) + (w & ((1u << a.share) - 1)));
}
// row `srow` of digit j at s, in order
template <uint32_t BETA>
__device__ __forceinline__ void pos_digit(const DevTables &c, const PosArgs &a, const PosRow &p, const u64 *ct, uint32_t srow, uint32_t j, double *s) {
    if (j == p.own) {
        const u64 *d = ct + p.cc + srow * 256 + 2 * p.t;
        ulonglong2 w[4];
#pragma unroll
        for (uint32_t k = 0; k < 4; k++) w[k] = ld_pair<true>(d + 64 * k);
#pragma unroll
        for (uint32_t k = 0; k < 4; k++) *reinterpret_cast<double2 *>(s + wrow_at(2 * p.t) + 72 * k) = make_double2(u64_to_d(w[k].x), u64_to_d(w[k].y));
        return;
    }
    const double *g = reinterpret_cast<const double *>(a.ext) + (((size_t)p.bz * BETA + j) * p.nt + p.x) * p.limb + srow * 256 + p.t;
    double v[8];
#pragma unroll
    for (uint32_t k = 0; k < 8; k++) v[k] = g[32 * k];
    wrow_forward(v, s, p.t, c.twd_fwd + p.kt * p.limb, p.R + srow, p.q, p.qinv);
}
// the digits' rows `srow` in shared memory
template <uint32_t BETA>
__device__ __forceinline__ void pos_digits(const DevTables &c, const PosArgs &a, const PosRow &p, const u64 *ct, uint32_t srow, double (&sm)[BETA][MID_ROWS][WROW_PAD]) {
#pragma unroll 1
    for (uint32_t j = 0; j < BETA; j++) pos_digit<BETA>(c, a, p, ct, srow, j, sm[j][p.rl]);
    __syncwarp();
}
// e = S_r (<digits, key>_cm + [cm = 0] P sigma_r(c0)) of both components at the words p0 + 64 k, p0 + 64 k + 1: below 1.5 q
template <uint32_t BETA>
__device__ __forceinline__ void pos_pair(const DevTables &c, const PosArgs &a, const PosRow &p, const u64 *ct, uint32_t r, uint32_t k,
                                         const double (&sm)[BETA][MID_ROWS][WROW_PAD], double2 (&e)[2]) {
    const uint32_t gal = (uint32_t)a.galois[r], p0 = p.row * 256 + 2 * p.t + 64 * k, src = galois_src(p0, gal, c.log_n), so = src & 254u;
    const bool odd = src & 1;                // the permutation maps the pair onto a pair, possibly swapped
    const u64 *kp = a.evk[r] + p.kt * p.limb + p0;
    ulonglong2 kv[BETA][2], z = make_ulonglong2(0, 0);
#pragma unroll
    for (uint32_t j = 0; j < BETA; j++) {
        kv[j][0] = ld_pair<true>(kp + 2 * j * p.kc);
        kv[j][1] = ld_pair<true>(kp + (2 * j + 1) * p.kc);
    }
    const ulonglong2 f = ld_pair<true>(a.fac + r * a.fac_rot + p.set * a.fac_set + p.x * p.limb + p0);
    if (p.x < a.level) z = ld_pair<true>(ct + (src & ~1u));
    // products of the own digit and of c0 below q^2, of the other three at most below q^2 / 2: below 4 q^2 in all
    ProductSum s00, s01, s10, s11;
    s00.add(u64_to_d(odd ? z.y : z.x), p.pq);
    s01.add(u64_to_d(odd ? z.x : z.y), p.pq);
#pragma unroll
    for (uint32_t j = 0; j < BETA; j++) {
        const double2 d = *reinterpret_cast<const double2 *>(sm[j][p.rl] + wrow_at(so));
        const double d0 = odd ? d.y : d.x, d1 = odd ? d.x : d.y;
        s00.add(d0, u64_to_d(kv[j][0].x)); s01.add(d1, u64_to_d(kv[j][0].y));
        s10.add(d0, u64_to_d(kv[j][1].x)); s11.add(d1, u64_to_d(kv[j][1].y));
    }
    const double f0 = u64_to_d(f.x), f1 = u64_to_d(f.y);
    e[0] = make_double2(mulmod_pq<1>(s00.sum(p.q, p.qinv), f0, p.q, p.qinv), mulmod_pq<1>(s01.sum(p.q, p.qinv), f1, p.q, p.qinv));
    e[1] = make_double2(mulmod_pq<1>(s10.sum(p.q, p.qinv), f0, p.q, p.qinv), mulmod_pq<1>(s11.sum(p.q, p.qinv), f1, p.q, p.qinv));
}
// P C c of both components there: below 0.75 q
__device__ __forceinline__ void pos_own(const PosArgs &a, const PosRow &p, const u64 *ct, uint32_t k, double2 (&o)[2]) {
    o[0] = o[1] = make_double2(0.0, 0.0);
    if (p.x >= a.level) return;
    const uint32_t p0 = p.row * 256 + 2 * p.t + 64 * k;
    const ulonglong2 w = ld_pair<true>(a.own + p.set * a.own_set + p.x * p.limb + p0), z0 = ld_pair<true>(ct + p0), z1 = ld_pair<true>(ct + p.cc + p0);
    const double w0 = mulmod_dd(u64_to_d(w.x), p.pq, p.q, p.qinv), w1 = mulmod_dd(u64_to_d(w.y), p.pq, p.q, p.qinv);
    o[0] = make_double2(mulmod_dd(u64_to_d(z0.x), w0, p.q, p.qinv), mulmod_dd(u64_to_d(z0.y), w1, p.q, p.qinv));
    o[1] = make_double2(mulmod_dd(u64_to_d(z1.x), w0, p.q, p.qinv), mulmod_dd(u64_to_d(z1.y), w1, p.q, p.qinv));
}
// the row's words p0 + 64 k, p0 + 64 k + 1 in v, at most half a prime -> the inverse row pass's result in g
__device__ __forceinline__ void pos_inverse(const DevTables &c, const PosRow &p, double (&v)[8], double *s, double *g) {
#pragma unroll
    for (uint32_t k = 0; k < 4; k++) *reinterpret_cast<double2 *>(s + wrow_at(2 * p.t) + 72 * k) = make_double2(v[2 * k], v[2 * k + 1]);
    __syncwarp();
    wrow_inverse(v, s, p.t, c.twd_inv + p.kt * p.limb, p.R + p.row, p.q, p.qinv);
#pragma unroll
    for (uint32_t k = 0; k < 8; k++) g[p.t + 32 * k] = v[k];
    __syncwarp();
}

// Pair by pair, nothing is held from one to the next: the sums of all rotations but the last (MANY) and the pairs of a limb that is transformed
// back wait in their place in u.  One ciphertext at level 18: 42 us; two rotations of six at N = 2^15, level 10: 98 us, where sums kept in registers, and
// five CTAs per SM with them, took 103.
template <uint32_t BETA, bool MANY>
__global__ void __launch_bounds__(32 * MID_ROWS, 6) mid_rows_pos(DevTables c, const __grid_constant__ PosArgs a) {
    __shared__ __align__(16) double sm[BETA][MID_ROWS][WROW_PAD];
    const PosRow p = pos_warp(c, a, BETA);
    grid_dep_sync();
    if (p.bz >= a.nb) return;
    const u64 *ct = a.c.at(p.bz) + p.x * p.limb;
    u64 *u0 = a.u + ((size_t)p.bz * 2 * p.nt + p.x) * p.limb + p.row * 256;
    const bool inverse = p.x >= a.inv_from;
#pragma unroll 1
    for (uint32_t r = 0; r < (MANY ? a.nrot : 1); r++) {
        pos_digits<BETA>(c, a, p, ct, galois_src(p.row << 8, (uint32_t)a.galois[r], c.log_n) >> 8, sm);
        const bool last = !MANY || r + 1 == a.nrot;
#pragma unroll
        for (uint32_t k = 0; k < 4; k++) {
            u64 *u = u0 + 2 * p.t + 64 * k;
            double2 e[2], o[2];
            pos_pair<BETA>(c, a, p, ct, r, k, sm, e);
            if (MANY && r)           // below 1.5 q per rotation
#pragma unroll
                for (uint32_t cm = 0; cm < 2; cm++) o[cm] = *reinterpret_cast<const double2 *>(u + cm * p.nt * p.limb);
            else pos_own(a, p, ct, k, o);
#pragma unroll
            for (uint32_t cm = 0; cm < 2; cm++) {
                double x = __dadd_rn(e[cm].x, o[cm].x), y = __dadd_rn(e[cm].y, o[cm].y);
                if (last) { x = reduce_d(x, p.q, p.qinv); y = reduce_d(y, p.q, p.qinv); }
                if (inverse || !last) *reinterpret_cast<double2 *>(u + cm * p.nt * p.limb) = make_double2(x, y);
                else st_pair<true>(u + cm * p.nt * p.limb, make_ulonglong2(canonical_d(x, p.q), canonical_d(y, p.q)));
            }
            asm volatile("" ::: "memory");       // one step's words at a time: the registers hold no more
        }
        if (MANY) __syncwarp();
    }
    if (!inverse) return;
#pragma unroll 1
    for (uint32_t cm = 0; cm < 2; cm++, u0 += p.nt * p.limb) {
        double v[8];
#pragma unroll
        for (uint32_t k = 0; k < 4; k++) {
            const double2 w = *reinterpret_cast<const double2 *>(u0 + 2 * p.t + 64 * k);
            v[2 * k] = w.x; v[2 * k + 1] = w.y;
        }
        __syncwarp();
        pos_inverse(c, p, v, sm[0][p.rl], reinterpret_cast<double *>(u0));
    }
}

// Five to eight digits: a CTA per row, a warp per digit, then the row's pairs of both components over all threads, because one warp would
// transform the digits one after the other (one ciphertext at N = 2^13, six digits: 47 us for the call, 41 with launches of their own for the
// transforms and positions_inner, 37 so; wide_rows in positions.cu says up to where).  With three digits it is slower from the first ciphertext on at
// N = 2^16 (180 -> 212 us for a token's append) and little faster at N = 2^14 (86 -> 84).
template <uint32_t BETA>
__global__ void __launch_bounds__(32 * BETA) mid_rows_pos_wide(DevTables c, const __grid_constant__ PosArgs a) {
    constexpr uint32_t THREADS = 32 * BETA, ITEMS = (256 + THREADS - 1) / THREADS;
    __shared__ __align__(16) double sm[BETA][WROW_PAD];
    const PosRow p = pos_row(c, a, BETA, blockIdx.x, blockIdx.y);
    double2 acc[ITEMS];                 // item: pair 0 .. 127 of component 0, then of component 1
    grid_dep_sync();
    const u64 *ct = a.c.at(p.bz) + p.x * p.limb;
#pragma unroll
    for (uint32_t i = 0; i < ITEMS; i++) {
        const uint32_t w = threadIdx.x + i * THREADS, at = p.row * 256 + 2 * (w & 127), cm = w >> 7;
        acc[i] = make_double2(0.0, 0.0);
        if (w >= 256 || p.x >= a.level) continue;
        const ulonglong2 o = ld_pair<true>(a.own + p.set * a.own_set + p.x * p.limb + at), z = ld_pair<true>(ct + cm * p.cc + at);
        acc[i] = make_double2(mulmod_dd(mulmod_dd(u64_to_d(z.x), u64_to_d(o.x), p.q, p.qinv), p.pq, p.q, p.qinv),
                              mulmod_dd(mulmod_dd(u64_to_d(z.y), u64_to_d(o.y), p.q, p.qinv), p.pq, p.q, p.qinv));
    }
#pragma unroll 1
    for (uint32_t r = 0; r < a.nrot; r++) {
        const uint32_t gal = (uint32_t)a.galois[r];
        pos_digit<BETA>(c, a, p, ct, galois_src(p.row << 8, gal, c.log_n) >> 8, p.rl, sm[p.rl]);
        __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < ITEMS; i++) {
            const uint32_t w = threadIdx.x + i * THREADS, at = p.row * 256 + 2 * (w & 127), cm = w >> 7;
            if (w >= 256) continue;
            const uint32_t src = galois_src(at, gal, c.log_n), so = src & 254u;
            const bool odd = src & 1;                // the permutation maps the pair onto a pair, possibly swapped
            const u64 *kp = a.evk[r] + cm * p.kc + p.kt * p.limb + at;
            ulonglong2 kv[BETA];
#pragma unroll
            for (uint32_t j = 0; j < BETA; j++) kv[j] = ld_pair<true>(kp + 2 * j * p.kc);
            const ulonglong2 f = ld_pair<true>(a.fac + r * a.fac_rot + p.set * a.fac_set + p.x * p.limb + at);
            // as in pos_pair; the sum of c0's product and four digits' is reduced before the others'
            ProductSum e0, e1;
            if (cm == 0 && p.x < a.level) {
                const ulonglong2 z = ld_pair<true>(ct + (src & ~1u));
                e0.add(u64_to_d(odd ? z.y : z.x), p.pq);
                e1.add(u64_to_d(odd ? z.x : z.y), p.pq);
            }
#pragma unroll
            for (uint32_t j = 0; j < BETA; j++) {
                if (j == 4) { e0.carry(p.q, p.qinv); e1.carry(p.q, p.qinv); }
                const double2 d = *reinterpret_cast<const double2 *>(sm[j] + wrow_at(so));
                e0.add(odd ? d.y : d.x, u64_to_d(kv[j].x));
                e1.add(odd ? d.x : d.y, u64_to_d(kv[j].y));
            }
            acc[i].x = __dadd_rn(acc[i].x, mulmod_pq<1>(e0.sum(p.q, p.qinv), u64_to_d(f.x), p.q, p.qinv));
            acc[i].y = __dadd_rn(acc[i].y, mulmod_pq<1>(e1.sum(p.q, p.qinv), u64_to_d(f.y), p.q, p.qinv));
        }
        __syncthreads();
    }
    u64 *u = a.u + ((size_t)p.bz * 2 * p.nt + p.x) * p.limb + p.row * 256;
    const bool inverse = p.x >= a.inv_from;
#pragma unroll
    for (uint32_t i = 0; i < ITEMS; i++) {
        const uint32_t w = threadIdx.x + i * THREADS, at = 2 * (w & 127), cm = w >> 7;
        if (w >= 256) continue;
        const double x = reduce_d(acc[i].x, p.q, p.qinv), y = reduce_d(acc[i].y, p.q, p.qinv);
        if (inverse) *reinterpret_cast<double2 *>(sm[cm] + wrow_at(at)) = make_double2(x, y);
        else st_pair<true>(u + cm * p.nt * p.limb + at, make_ulonglong2(canonical_d(x, p.q), canonical_d(y, p.q)));
    }
    if (!inverse) return;
    __syncthreads();
    if (p.rl >= 2) return;
    double v[8];
    wrow_inverse(v, sm[p.rl], p.t, c.twd_inv + p.kt * p.limb, p.R + p.row, p.q, p.qinv);
    double *g = reinterpret_cast<double *>(u + p.rl * p.nt * p.limb) + p.t;
#pragma unroll
    for (uint32_t k = 0; k < 8; k++) g[32 * k] = v[k];
}

}  // namespace

void launch_mid_rows_pos(const ckks_ctx *c, const PosArgs &a, uint32_t beta, cudaStream_t s) {
    using K = decltype(&mid_rows_pos<1, false>);
    static constexpr K one[IP_FUSED_BETA] = {mid_rows_pos<1, false>, mid_rows_pos<2, false>, mid_rows_pos<3, false>, mid_rows_pos<4, false>};
    static constexpr K many[IP_FUSED_BETA] = {mid_rows_pos<1, true>, mid_rows_pos<2, true>, mid_rows_pos<3, true>, mid_rows_pos<4, true>};
    static constexpr K wide[POS_BETA - IP_FUSED_BETA] = {mid_rows_pos_wide<5>, mid_rows_pos_wide<6>, mid_rows_pos_wide<7>, mid_rows_pos_wide<8>};
    if (beta > IP_FUSED_BETA) {
        launch(wide[beta - 1 - IP_FUSED_BETA], dim3(c->N >> 8, a.nb, a.level + c->K), 32 * beta, 0, s, c->dev, a);
        return;
    }
    PosArgs b = a;
    // entries of a row in a CTA: few idle warps, so groups that they fill, or many groups.  Rotation at N = 2^16, level 24, in ones / twos / fours, us: one
    // ciphertext 188 / 206 / 241, two 292 / 291 / 321, three 416 / 416 / 417, four 544 / 531 / 531, five 638 / 640 / 660, six 747 / 738 / 756, eight
    // 954 / 944 / 939, twelve 1391 / 1376 / 1367, thirteen 1510 / 1510 / 1508, sixteen 1808 / 1787 / 1789
    b.share = a.nb % 4 == 0 || a.nb > 12 ? 2 : a.nb % 2 == 0 || a.nb > 4 ? 1 : 0;
    const uint32_t e = 1u << b.share;
    launch((a.nrot > 1 ? many : one)[beta - 1], dim3((c->N >> 8) / (MID_ROWS >> b.share), (a.nb + e - 1) / e, a.level + c->K), 32 * MID_ROWS, 0, s, c->dev, b);
}
void launch_mid_rows(const ckks_ctx *c, const MidArgs &a, uint32_t beta, cudaStream_t s) {
    using K = decltype(&mid_rows<1, false>);
    static constexpr K one[IP_FUSED_BETA] = {mid_rows<1, false>, mid_rows<2, false>, mid_rows<3, false>, mid_rows<4, false>};
    static constexpr K terms[IP_FUSED_BETA] = {mid_rows<1, true>, mid_rows<2, true>, mid_rows<3, true>, mid_rows<4, true>};
    launch((a.nterm > 1 || a.c0[0] ? terms : one)[beta - 1], dim3((c->N >> 8) / MID_ROWS, a.nb, a.level + c->K), 32 * MID_ROWS, 0, s, c->dev, a);
}
