// Positions of a decoder's tokens on ciphertexts in the projections' token-shard layout: the table of angles, the rotation of queries and
// keys by it, and the append of new keys (rotated on the way) and values to a cache of pages, a page being the shard ciphertext of
// token_inner neighbouring tokens.
//
// Rotation.  Slot ((copy dim + d) heads + h) token_inner + t holds channel d.  Channel d of a pair gets cos x_d -/+ sin x_partner, the
// partner `apart` channels away (half of the rotated channels, or the neighbour):
//     out = rescale( C x + sum_r S_r rot_r(x) ),      r = +apart and -apart channels (one cyclic rotation where apart is half a head).
// The products by S_r are taken in the key-switching basis, before the division by P, which all rotations then share and which ends in
// the rescale (ks_down_rescale):   U = sum_r S_r (<ModUp(c1) read through sigma_r, key_r> + P sigma_r(c0)) + P C c,
// out = U / (P q_{l-1}).  Per ciphertext that takes the transforms of one key switch and two of a dropped limb, where a rotation, products
// and a rescale after one another take 48 more at level 24; digits are formed once however many rotations there are.
// Plaintexts are encoded from the table where the encoder reads its slots, once for all ciphertexts of a call that share their positions.
#include <map>
#include <tuple>
#include <vector>

#include "common.cuh"
#include "frequencies.cuh"

namespace {

constexpr uint32_t THREADS = 256;

// ---- the table of angles --------------------------------------------------------------------------------------------
constexpr uint32_t ROT_MAX = 256;
struct Turns { double hi[ROT_MAX / 2], lo[ROT_MAX / 2]; };      // angle per position over pi, as an unevaluated sum (frequencies.cuh)

// The angle over pi is formed as a sum of two doubles and reduced exactly, so that far positions lose nothing.  A unit is off by less
// than 3 * 2^-52: by its argument's rounding, at most pi 2^-53, and by two units in the last place of each of its values.
__device__ __forceinline__ double2 unit(double pos, double w_hi, double w_lo) {
    const double hi = __dmul_rn(pos, w_hi), lo = __fma_rn(pos, w_lo, __fma_rn(pos, w_hi, -hi));
    const double r = __dsub_rn(hi, __dmul_rn(2.0, rint(__dmul_rn(0.5, hi))));
    double s, c;
    sincospi(__dadd_rn(r, lo), &s, &c);
    return make_double2(c, s);
}
// cos, sin [count][half] of position first + row, a CTA per R^2 rows and 32 columns: R + R units per column from the functions, the others
// as products e^(i w (base + offset)), four operations where the function takes tens.  Their error is that of two units, of the
// magnitude's product and of their own: below 7 * 2^-52 times the magnitude, and 2^-52 from the frequency at position 2^50.  Bound by its
// stores from R = 16 on: 131072 positions of 64 pairs, 134 MB, in 24.9 us (5.4 TB/s; 121 us with every value from the function).
template <uint32_t R>
__global__ void __launch_bounds__(THREADS) rotary_table_kernel(const __grid_constant__ Turns w, uint64_t first, uint64_t count, uint32_t half, double magnitude,
                                                             double *cosv, double *sinv) {
    __shared__ double2 base[R][32], off[R][32];
    const uint32_t col = threadIdx.x & 31, j = blockIdx.y * 32 + col, g = threadIdx.x >> 5;
    const uint64_t row0 = (uint64_t)blockIdx.x * (R * R);
    grid_dep_sync();
    if (j < half)
        for (uint32_t x = g; x < R; x += THREADS / 32) {
            const double2 b = unit((double)(first + row0 + x * R), w.hi[j], w.lo[j]);
            base[x][col] = make_double2(__dmul_rn(b.x, magnitude), __dmul_rn(b.y, magnitude));
            off[x][col] = unit((double)x, w.hi[j], w.lo[j]);
        }
    __syncthreads();
    if (j >= half) return;
    for (uint32_t y = g; y < R; y += THREADS / 32) {
        const double2 o = off[y][col];
#pragma unroll 4
        for (uint32_t x = 0; x < R; x++) {
            const uint64_t row = row0 + x * R + y;
            if (row >= count) break;
            const double2 b = base[x][col];
            const size_t at = row * half + j;
            cosv[at] = __fma_rn(b.x, o.x, -__dmul_rn(b.y, o.y));
            sinv[at] = __fma_rn(b.x, o.y, __dmul_rn(b.y, o.x));
        }
    }
}

// ---- PosArgs' sums for any number of digits and any alignment: one coefficient of both components per thread, bound by its 8-byte loads
__global__ void __launch_bounds__(THREADS) positions_inner(DevTables c, const __grid_constant__ PosArgs a) {
    const uint32_t p = blockIdx.x * THREADS + threadIdx.x, bz = blockIdx.y, x = blockIdx.z;
    const uint32_t nt = a.level + c.K, beta = (a.level + c.alpha - 1) / c.alpha, kt = x < a.level ? x : c.L + (x - a.level);
    const uint32_t own = x < a.level ? x / c.alpha : beta, set = a.set[bz];
    const double q = c.modd[kt].x, qinv = c.modd[kt].y, pq = x < a.level ? c.dn_p_mod_d[x] : 0.0;
    const size_t limb = (size_t)1 << c.log_n, cc = a.pitch * limb;
    grid_dep_sync();
    const u64 *ct = a.c.at(bz) + x * limb, *ext = a.ext + ((size_t)bz * beta * nt + x) * limb;
    double s0 = 0.0, s1 = 0.0;
    for (uint32_t r = 0; r < a.nrot; r++) {
        const uint32_t src = galois_src(p, (uint32_t)a.galois[r], c.log_n);
        double e0 = x < a.level ? mulmod_dd(u64_to_d(ct[src]), pq, q, qinv) : 0.0, e1 = 0.0;
        for (uint32_t j = 0; j < beta; j++) {
            const double d = u64_to_d(j == own ? ct[cc + src] : ext[j * nt * limb + src]);
            const u64 *k = a.evk[r] + ((size_t)2 * j * c.T + kt) * limb + p;
            e0 = __dadd_rn(e0, mulmod_dd(d, u64_to_d(k[0]), q, qinv));
            e1 = __dadd_rn(e1, mulmod_dd(d, u64_to_d(k[c.T * limb]), q, qinv));
            if ((j & 7) == 7) { e0 = reduce_d(e0, q, qinv); e1 = reduce_d(e1, q, qinv); }
        }
        const double f = u64_to_d(a.fac[r * a.fac_rot + set * a.fac_set + x * limb + p]);
        s0 = __dadd_rn(s0, mulmod_dd(reduce_d(e0, q, qinv), f, q, qinv));
        s1 = __dadd_rn(s1, mulmod_dd(reduce_d(e1, q, qinv), f, q, qinv));
    }
    if (x < a.level) {
        const double w = u64_to_d(a.own[set * a.own_set + x * limb + p]);
        s0 = __dadd_rn(s0, mulmod_dd(mulmod_dd(u64_to_d(ct[p]), w, q, qinv), pq, q, qinv));
        s1 = __dadd_rn(s1, mulmod_dd(mulmod_dd(u64_to_d(ct[cc + p]), w, q, qinv), pq, q, qinv));
    }
    u64 *u = a.u + ((size_t)bz * 2 * nt + x) * limb + p;
    u[0] = canonical_d(reduce_d(s0, q, qinv), q);
    u[nt * limb] = canonical_d(reduce_d(s1, q, qinv), q);
}

// out = a + b, b's components b_pitch limbs apart, of nb two-component ciphertexts (a page and the tokens that fill it)
template <bool WIDE>
__global__ void __launch_bounds__(THREADS) add_pages(DevTables c, const __grid_constant__ Ptrs a, const __grid_constant__ Ptrs b, const __grid_constant__ Ptrs out, uint32_t level,
                                                     uint32_t b_pitch) {
    const uint32_t p = (blockIdx.x * THREADS + threadIdx.x) * 2, i = blockIdx.y, z = blockIdx.z >> 1, comp = blockIdx.z & 1;
    const u64 q = c.mod[i];
    const size_t at = (((size_t)comp * level + i) << c.log_n) + p;
    grid_dep_sync();
    const ulonglong2 u = ld_pair<WIDE>(a.at(z) + at), v = ld_pair<WIDE>(b.at(z) + (((size_t)comp * b_pitch + i) << c.log_n) + p);
    st_pair<WIDE>(const_cast<u64 *>(out.at(z)) + at, make_ulonglong2(add_mod(u.x, v.x, q), add_mod(u.y, v.y, q)));
}

// ---- shapes ------------------------------------------------------------------------------------------------------------
struct RotaryPlan {
    uint32_t nrot;
    int64_t rots[POS_ROT];
};

int make_plan(const ckks_ctx *c, const ckks_rotary_desc *d, RotaryPlan &p) {
    if (!d || !d->dim || !d->heads || !d->token_inner || !d->rot_dim || d->row_step > 1) return CKKS_ERR_ARG;
    if (d->layout != CKKS_ROTARY_HALF && d->layout != CKKS_ROTARY_INTERLEAVED) return CKKS_ERR_ARG;
    if ((d->rot_dim & 1) || d->rot_dim > d->dim) return CKKS_ERR_UNSUPPORTED;
    if (d->dim > c->n || d->heads > c->n || d->token_inner > c->n) return CKKS_ERR_UNSUPPORTED;
    const uint64_t period = (uint64_t)d->dim * d->heads;           // at most 2^30
    if (period > c->n || period * d->token_inner > c->n || c->n % (period * d->token_inner)) return CKKS_ERR_UNSUPPORTED;
    const uint32_t apart = d->layout == CKKS_ROTARY_HALF ? d->rot_dim / 2 : 1;
    p.nrot = 2 * apart == d->dim ? 1 : 2;
    p.rots[0] = (int64_t)apart * d->heads * d->token_inner;
    p.rots[1] = -p.rots[0];
    return CKKS_OK;
}

const ckks_evk *find_key(const ckks_ctx *c, const ckks_evk *keys, uint32_t nkeys, int64_t rot) {
    const uint64_t g = ckks_galois_element(c, rot);
    for (uint32_t i = 0; i < nkeys && keys; i++)
        if (keys[i].galois == g && keys[i].data) return &keys[i];
    return nullptr;
}

// Calls of a few ciphertexts on large rings, whose launches leave most of the GPU idle, run what does not depend on each other side by side: the
// plaintexts' encoding next to the extension of the digits, the values next to the keys.  An append on one stream / on two, us: N = 2^16, level 18,
// one ciphertext 215 / 187, two 355 / 327, four 657 / 634, eight 1192 / 1181, sixteen 2304 / 2310; N = 2^15, level 10, one 91 / 81, four 191 / 169,
// eight 336 / 308, sixteen 621 / 589; a rotation gains at most 10 (166 / 156).  On smaller rings the fork's events cost the host of a short call
// what the GPU gains, or more: N = 2^13, level 6, one 59.1 / 61.1, two 71.4 / 73.0, eight 109 / 112; N = 2^14, one 58.2 / 60.5, two 63.7 / 63.7.
// (The same calls from a graph, 48 / 33, 53 / 39, 96 / 82 and 55 / 40, 63 / 55, and from four on at N = 2^14, 84 / 80, would gain; the rule looks
// at the ring and the number alone.)
bool side_by_side(const ckks_ctx *c, uint32_t n) { return c->log_n >= 15 && n <= (4u << (16 - c->log_n)); }

// mid_rows_pos_wide takes the rows of five to eight digits while its CTAs, one per row, are few: 25 per SM with one rotation, 10 with two, for which
// it transforms the digits twice and plain transforms before positions_inner once.  Call, us, with launches apart / with it: six digits at N = 2^13, one
// rotation, one ciphertext 42 / 38, eight 68 / 63, sixteen 106 / 104; at N = 2^14 eight 112 / 110, sixteen 187 / 191; two rotations at N = 2^13, one 44 / 40,
// six 70 / 67, eight 77 / 78, sixteen 122 / 131; eight digits at N = 2^13, two rotations, three 62.5 / 60.6, five 81 / 81, sixteen 176 / 193.  From
// N = 2^15 on launches apart fill the GPU from the first ciphertext: five digits, one rotation 65 / 69, two rotations 81 / 92, sixteen 588 / 704.
bool wide_rows(const ckks_ctx *c, uint32_t level, uint32_t nrot, uint32_t nb) {
    return c->log_n <= 14 && (uint64_t)(c->N >> 8) * nb * (level + c->K) <= (nrot == 1 ? 25 : 10) * (uint64_t)c->sms;
}

// Workspace of a pass over up to `m` sets of positions and `m` ciphertexts side by side: plaintexts, then the encoder's scratch, whose
// place the key switches take over (side by side: behind it), and after them the values'
struct RotaryWs { size_t rest, ks, values, bytes; };
RotaryWs rotary_ws(const ckks_ctx *c, uint32_t level, uint32_t nrot, bool mask, uint32_t m) {
    const size_t N = c->N * sizeof(u64), enc = align256(encode_workspace_bytes(c, m * (1 + nrot + mask))), ks = align256((size_t)m * ks_workspace_limbs(c, level) * N);
    RotaryWs w;
    w.rest = align256((size_t)m * (1 + nrot + mask) * (level + c->K) * N);
    if (!side_by_side(c, m)) {
        w.ks = w.values = w.rest;
        w.bytes = w.rest + std::max(enc, ks);
        return w;
    }
    w.ks = w.rest + enc;
    w.values = w.ks + ks;
    w.bytes = w.values + (mask ? align256(plain_rescale_limbs(level, m) * N) : 0);
    return w;
}
size_t rotary_bytes(const ckks_ctx *c, uint32_t level, uint32_t nrot, bool mask, uint32_t m) { return rotary_ws(c, level, nrot, mask, m).bytes; }
size_t mask_bytes(const ckks_ctx *c, uint32_t level, uint32_t m) {
    const size_t N = c->N * sizeof(u64);
    return align256((size_t)m * level * N) + align256(std::max(encode_workspace_bytes(c, m), plain_rescale_limbs(level, m) * N));
}

// One ciphertext's share: where it is read and written, what is added, the positions of its tokens
struct Item {
    const u64 *in, *acc;
    u64 *out;
    uint32_t row, begin, end;
};

// The rotation of items read at `level` (components `pitch` limbs apart), written at level - 1.  Items of the same positions share their
// plaintexts; up to SLOT_SETS sets are encoded at a time.  values (may be null): as many items, appended under the mask of their item's span,
// which is encoded with the set (four launches less: one token's append at N = 2^16, level 18, 230 -> 213 us).
void rotate_items(ckks_ctx *c, const ckks_rotary_desc *d, const RotaryPlan &p, const std::vector<Item> &items, uint32_t pitch, uint32_t level, const double *cosv,
                  const double *sinv, const ckks_evk *keys, uint32_t nkeys, void *ws, cudaStream_t s, const std::vector<Item> *values = nullptr, uint32_t values_pitch = 0) {
    std::map<std::tuple<uint32_t, uint32_t, uint32_t>, std::vector<uint32_t>> by;
    std::vector<std::vector<uint32_t>> sets;
    for (uint32_t i = 0; i < items.size(); i++) {
        auto &v = by[std::make_tuple(items[i].row, items[i].begin, items[i].end)];
        v.push_back(i);
    }
    for (auto &e : by) sets.push_back(std::move(e.second));
    const size_t N = c->N;
    const uint32_t nt = level + c->K, beta = (level + c->alpha - 1) / c->alpha, m = std::min((uint32_t)items.size(), KS_MULTI);
    const double scale = (double)c->mod[level - 1];
    const uint32_t kinds = 1 + p.nrot + (values ? 1 : 0);        // a set: C, the S_r, the mask, each level + K limbs apart
    const RotaryWs at = rotary_ws(c, level, p.nrot, values != nullptr, m);
    u64 *pts = (u64 *)ws;
    void *rest = (char *)ws + at.rest, *ksw = (char *)ws + at.ks, *vws = (char *)ws + at.values;
    // lane 1 (the caller's stream where the call does not fork): plaintexts, then the values
    Lanes lanes(c, s, side_by_side(c, (uint32_t)items.size()));
    const bool fork = lanes.n > 1;
    cudaStream_t side = fork ? (cudaStream_t)lanes.at(1) : s;
    if (fork) lanes.fork(1);
    for (uint32_t s0 = 0; s0 < sets.size(); s0 += SLOT_SETS) {
        const uint32_t ns = std::min(SLOT_SETS, (uint32_t)sets.size() - s0);
        SlotPositions slots{cosv, sinv, log2_of(d->dim), log2_of(d->heads), log2_of(d->token_inner), d->rot_dim, d->layout == CKKS_ROTARY_INTERLEAVED, d->row_step, p.nrot, kinds, {}, {}, {}};
        std::vector<std::pair<uint32_t, uint32_t>> todo;               // (item, set)
        for (uint32_t k = 0; k < ns; k++) {
            const Item &it = items[sets[s0 + k][0]];
            slots.row[k] = it.row; slots.begin[k] = it.begin; slots.end[k] = it.end;
            for (uint32_t i : sets[s0 + k]) todo.emplace_back(i, k);
        }
        const uint32_t batch = ns * kinds;
        launch_encode_slots(c, slots, batch, scale, rest, side);
        launch_encode_coefs(c, rest, batch, batch * nt, set_map(level, p.nrot, kinds, c->K, c->L), pts, side, true);
        if (fork) lanes.mark(1);
        for (size_t i0 = 0; i0 < todo.size(); i0 += KS_MULTI) {
            const uint32_t nb = (uint32_t)std::min<size_t>(KS_MULTI, todo.size() - i0);
            KsWorkspace w = ks_carve(c, level, ksw, nb);
            w.alone = items.size() == 1;
            PosArgs a{};
            Ptrs c1, out, acc;
            a.c.n = c1.n = out.n = acc.n = nb;
            for (uint32_t b = 0; b < nb; b++) {
                const Item &it = items[todo[i0 + b].first];
                a.set[b] = (uint8_t)todo[i0 + b].second;
                a.c.p[b] = it.in; c1.p[b] = it.in + pitch * N;
                out.p[b] = it.out; acc.p[b] = it.acc;
            }
            for (uint32_t r = 0; r < p.nrot; r++) {
                const ckks_evk *k = find_key(c, keys, nkeys, p.rots[r]);
                a.evk[r] = (const u64 *)k->data; a.galois[r] = k->galois;
            }
            w.mid = ks_mid(c, level, w, c1, a.evk, p.nrot, wide_rows(c, level, p.nrot, nb) ? POS_BETA : IP_FUSED_BETA) && aligned16(a.c) && aligned16(pts);
            auto append_values = [&]() {
                PlainRescale v{};
                v.in.n = v.pt.n = v.acc.n = v.out.n = nb;
                v.pitch = values_pitch; v.acc_pitch = level - 1; v.level = level; v.add = true;
                for (uint32_t b = 0; b < nb; b++) {
                    const Item &it = (*values)[todo[i0 + b].first];
                    v.in.p[b] = it.in; v.acc.p[b] = it.acc; v.out.p[b] = it.out;
                    v.pt.p[b] = pts + (todo[i0 + b].second * (size_t)kinds + kinds - 1) * nt * N;
                }
                launch_plain_rescale(c, v, (u64 *)vws, side, nb);
            };
            if (values && !fork) append_values();        // its scratch is the key switches'
            ks_modup(c, c1, level, w, s, nb);
            if (values && fork) append_values();
            a.ext = w.ext; a.u = w.u; a.own = pts; a.fac = pts + (size_t)nt * N;
            a.own_set = a.fac_set = (size_t)kinds * nt * N; a.fac_rot = (size_t)nt * N;
            a.pitch = pitch; a.nrot = p.nrot; a.nb = nb; a.level = level; a.inv_from = level - 1;
            if (fork) lanes.wait(1);
            if (w.mid) launch_mid_rows_pos(c, a, beta, s);
            else launch(positions_inner, dim3(c->N / THREADS, nb, nt), THREADS, 0, s, c->dev, a);
            ks_down_rescale(c, level, w, out, items[0].acc ? &acc : nullptr, s, nb);
        }
    }
    lanes.join();
}

// Values (or keys without positions): tokens that fill their page are added as they are, others under a mask
void append_items(ckks_ctx *c, uint32_t token_inner, const std::vector<Item> &items, uint32_t pitch, uint32_t level, void *ws, cudaStream_t s) {
    const size_t N = c->N;
    std::vector<Item> whole, part;
    for (const Item &it : items) (it.begin == 0 && it.end == token_inner ? whole : part).push_back(it);
    const uint32_t m = std::min((uint32_t)items.size(), KS_MULTI);
    u64 *pts = (u64 *)ws;
    void *rest = (char *)ws + align256((size_t)m * level * N * sizeof(u64));
    for (size_t i0 = 0; i0 < whole.size(); i0 += KS_MULTI) {
        Ptrs a, b, o;
        a.n = b.n = o.n = (uint32_t)std::min<size_t>(KS_MULTI, whole.size() - i0);
        for (uint32_t i = 0; i < a.n; i++) { a.p[i] = whole[i0 + i].acc; b.p[i] = whole[i0 + i].in; o.p[i] = whole[i0 + i].out; }
        const bool wide = aligned16(a) && aligned16(b) && aligned16(o);
        launch(wide ? add_pages<true> : add_pages<false>, dim3(c->N / (2 * THREADS), level - 1, 2 * a.n), THREADS, 0, s, c->dev, a, b, o, level - 1, pitch);
    }
    for (size_t i0 = 0; i0 < part.size(); i0 += KS_MULTI) {
        const uint32_t nb = (uint32_t)std::min<size_t>(KS_MULTI, part.size() - i0);
        SlotTokens slots{log2_of(token_inner), {}, {}};
        PlainRescale pr{};
        pr.in.n = pr.acc.n = pr.out.n = nb;
        pr.pt = Ptrs(pts, level * N);
        pr.pitch = pitch; pr.acc_pitch = level - 1; pr.level = level; pr.add = true;
        for (uint32_t i = 0; i < nb; i++) {
            const Item &it = part[i0 + i];
            slots.begin[i] = it.begin; slots.end[i] = it.end;
            pr.in.p[i] = it.in; pr.acc.p[i] = it.acc; pr.out.p[i] = it.out;
        }
        launch_encode_slots(c, slots, nb, (double)c->mod[level - 1], rest, s);
        launch_encode_coefs(c, rest, nb, nb * level, plain_map(0, level), pts, s);
        launch_plain_rescale(c, pr, (u64 *)rest, s, nb);
    }
}

// what the rotation reads besides its ciphertexts
void read_factors(const ckks_ctx *c, const ckks_rotary_desc *d, const RotaryPlan &p, const double *cosv, const double *sinv, uint32_t table_rows, const ckks_evk *keys,
                  uint32_t nkeys, Buffers &b) {
    const size_t table = (size_t)table_rows * (d->rot_dim / 2) * sizeof(double);
    b.read(cosv, table);
    b.read(sinv, table);
    for (uint32_t r = 0; r < p.nrot; r++) b.read(find_key(c, keys, nkeys, p.rots[r])->data, (size_t)c->dnum * 2 * c->T * c->N * sizeof(u64));
}

}  // namespace

extern "C" int32_t ckks_rotary_table(ckks_ctx *c, const ckks_rotary_scaling *f, uint64_t first, uint64_t count, double *cosv, double *sinv, void *stream) {
    if (!c || !f || !cosv || !sinv || !count || !f->rot_dim) return CKKS_ERR_ARG;
    if (!(f->theta > 1.0) || !isfinite(f->theta) || f->kind < 0 || f->kind > CKKS_ROTARY_RAMP) return CKKS_ERR_ARG;
    if (!isfinite(f->magnitude) || f->magnitude < 0.0) return CKKS_ERR_ARG;
    if (f->kind != CKKS_ROTARY_PLAIN && (!(f->factor >= 1.0) || !isfinite(f->factor))) return CKKS_ERR_ARG;
    const bool by_turns = f->kind == CKKS_ROTARY_BANDS || f->kind == CKKS_ROTARY_RAMP;
    const double few = f->turns_few > 0.0 ? f->turns_few : 1.0, many = f->turns_many > 0.0 ? f->turns_many : f->kind == CKKS_ROTARY_BANDS ? 4.0 : 32.0;
    if (by_turns && (!(f->original_length > 0.0) || !isfinite(f->original_length) || !(many > few) || !isfinite(many))) return CKKS_ERR_ARG;
    if ((f->rot_dim & 1) || f->rot_dim > ROT_MAX || (f->kind == CKKS_ROTARY_BASE && f->rot_dim < 4)) return CKKS_ERR_UNSUPPORTED;
    // positions are exact in doubles, and so are their products' high parts once reduced
    if (first > (1ull << 50) || count > (1ull << 38) || first + count > (1ull << 50)) return CKKS_ERR_UNSUPPORTED;
    const uintptr_t bytes = count * (f->rot_dim / 2) * sizeof(double), pc = (uintptr_t)cosv, ps = (uintptr_t)sinv;
    if (pc < ps + bytes && ps < pc + bytes) return CKKS_ERR_ARG;
    Turns w;
    rotary_frequencies(*f, few, many, w.hi, w.lo);
    const uint32_t half = f->rot_dim / 2, cols = (half + 31) / 32;
    const double mag = f->magnitude == 0.0 ? 1.0 : f->magnitude;
    DeviceGuard guard(c->device);
    // larger tiles once they give every SM two CTAs; below that the call is one launch's latency either way
    if (count / 256 * cols >= 2 * (uint64_t)c->sms)
        launch(rotary_table_kernel<16>, dim3((uint32_t)((count + 255) / 256), cols), THREADS, 0, (cudaStream_t)stream, w, first, count, half, mag, cosv, sinv);
    else
        launch(rotary_table_kernel<8>, dim3((uint32_t)((count + 63) / 64), cols), THREADS, 0, (cudaStream_t)stream, w, first, count, half, mag, cosv, sinv);
    return finish(c);
}

extern "C" int32_t ckks_rotary_rotations(const ckks_ctx *c, const ckks_rotary_desc *d, int64_t *rots, uint32_t cap) {
    if (!c) return CKKS_ERR_ARG;
    RotaryPlan p;
    const int rc = make_plan(c, d, p);
    if (rc) return rc;
    for (uint32_t r = 0; r < p.nrot && rots && r < cap; r++) rots[r] = p.rots[r];
    return (int32_t)p.nrot;
}

extern "C" size_t ckks_rotary_workspace_bytes(const ckks_ctx *c, const ckks_rotary_desc *d, uint32_t level, uint32_t n) {
    RotaryPlan p;
    if (!c || !n || level < 2 || level > c->L || make_plan(c, d, p)) return 0;
    return rotary_bytes(c, level, p.nrot, false, std::min(n, KS_MULTI));
}

extern "C" int32_t ckks_rotary(ckks_ctx *c, const ckks_rotary_desc *d, const ckks_ct *in, const uint32_t *rows, uint32_t n, const double *cosv, const double *sinv, uint32_t table_rows,
                               const ckks_evk *keys, uint32_t nkeys, ckks_ct *out, void *ws, size_t ws_bytes, void *stream) {
    if (!c || !in || !rows || !n || !cosv || !sinv || !out) return CKKS_ERR_ARG;
    return guarded(c, [&]() -> int32_t {
        RotaryPlan p;
        int rc = make_plan(c, d, p);
        if (rc) return rc;
        for (uint32_t i = 0; i < n; i++) {
            if (!in[i].data || in[i].ncomp != 2 || !out[i].data) return CKKS_ERR_ARG;
            if ((uint64_t)rows[i] + (uint64_t)(d->token_inner - 1) * d->row_step >= table_rows) return CKKS_ERR_ARG;
        }
        const uint32_t level = in[0].level;
        if (level < 2 || level > c->L) return CKKS_ERR_LEVEL;
        for (uint32_t i = 1; i < n; i++)
            if (in[i].level != level) return CKKS_ERR_LEVEL;
        const size_t bi = (size_t)2 * level * c->N * sizeof(u64), bo = (size_t)2 * (level - 1) * c->N * sizeof(u64);
        for (uint32_t r = 0; r < p.nrot; r++)
            if (!find_key(c, keys, nkeys, p.rots[r])) return CKKS_ERR_NO_KEY;
        const size_t need = rotary_bytes(c, level, p.nrot, false, std::min(n, KS_MULTI));
        if (!ws || ws_bytes < need) return CKKS_ERR_WORKSPACE;
        Buffers buffers;
        for (uint32_t i = 0; i < n; i++) { buffers.read(in[i].data, bi); buffers.write(out[i].data, bo); }
        read_factors(c, d, p, cosv, sinv, table_rows, keys, nkeys, buffers);
        buffers.write(ws, need);
        if (!buffers.apart()) return CKKS_ERR_ARG;
        std::vector<Item> items;
        for (uint32_t i = 0; i < n; i++) items.push_back(Item{(const u64 *)in[i].data, nullptr, (u64 *)out[i].data, rows[i], 0, d->token_inner});
        DeviceGuard guard(c->device);
        rotate_items(c, d, p, items, level, level, cosv, sinv, keys, nkeys, ws, (cudaStream_t)stream);
        rc = finish(c);
        for (uint32_t i = 0; i < n && rc == CKKS_OK; i++) { out[i].level = level - 1; out[i].ncomp = 2; out[i].scale = in[i].scale; }
        return rc;
    });
}

extern "C" size_t ckks_cache_append_workspace_bytes(const ckks_ctx *c, const ckks_rotary_desc *d, uint32_t page_level, uint32_t n) {
    RotaryPlan p;
    if (!c || !n || page_level < 1 || page_level >= c->L || make_plan(c, d, p)) return 0;
    const uint32_t m = std::min(n, KS_MULTI);
    return std::max(rotary_bytes(c, page_level + 1, p.nrot, true, m), mask_bytes(c, page_level + 1, m));
}

extern "C" int32_t ckks_cache_append(ckks_ctx *c, const ckks_rotary_desc *d, const ckks_ct *in_k, const ckks_ct *in_v, uint32_t n, const uint32_t *pages,
                                     const ckks_cache_span *spans, const ckks_ct *page_k, const ckks_ct *page_v, uint32_t npages, const double *cosv,
                                     const double *sinv, uint32_t table_rows, const ckks_evk *keys, uint32_t nkeys, ckks_ct *out_k, ckks_ct *out_v, void *ws, size_t ws_bytes,
                                     void *stream) {
    if (!c || !n || !pages || !spans || !npages || (!in_k && !in_v)) return CKKS_ERR_ARG;
    return guarded(c, [&]() -> int32_t {
        if ((in_k && (!page_k || !out_k)) || (in_v && (!page_v || !out_v)) || (!cosv) != (!sinv)) return CKKS_ERR_ARG;
        RotaryPlan p;
        int rc = make_plan(c, d, p);
        if (rc) return rc;
        const bool rotated = in_k && cosv;
        std::vector<uint32_t> named(pages, pages + n);
        std::sort(named.begin(), named.end());
        if (named.back() >= npages || std::adjacent_find(named.begin(), named.end()) != named.end()) return CKKS_ERR_ARG;
        for (uint32_t i = 0; i < n; i++) {
            if (spans[i].begin >= spans[i].end || spans[i].end > d->token_inner) return CKKS_ERR_ARG;
            if (rotated && (uint64_t)spans[i].row + (uint64_t)(spans[i].end - 1 - spans[i].begin) * d->row_step >= table_rows) return CKKS_ERR_ARG;
        }
        // descriptors: every side of the call on its own, then the buffers that are written against all others
        struct Side { const ckks_ct *in, *page; ckks_ct *out; uint32_t level, pitch; };
        std::vector<Side> sides;
        if (in_k) sides.push_back(Side{in_k, page_k, out_k, 0, 0});
        if (in_v) sides.push_back(Side{in_v, page_v, out_v, 0, 0});
        uint32_t level = 0;
        for (Side &sd : sides) {
            for (uint32_t i = 0; i < n; i++) {
                const ckks_ct &x = sd.in[i], &pg = sd.page[pages[i]];
                if (!x.data || x.ncomp != 2 || !pg.data || pg.ncomp != 2 || !sd.out[pages[i]].data) return CKKS_ERR_ARG;
            }
            sd.pitch = sd.in[0].level; sd.level = sd.page[pages[0]].level;
            if (!level) level = sd.level;
            if (sd.level < 1 || sd.level != level || sd.pitch <= level || sd.pitch > c->L) return CKKS_ERR_LEVEL;
            for (uint32_t i = 0; i < n; i++)
                if (sd.in[i].level != sd.pitch || sd.page[pages[i]].level != level) return CKKS_ERR_LEVEL;
            for (uint32_t i = 0; i < n; i++)
                if (!scales_agree(sd.in[i].scale, sd.page[pages[i]].scale)) return CKKS_ERR_SCALE;
        }
        for (uint32_t r = 0; r < p.nrot && rotated; r++)
            if (!find_key(c, keys, nkeys, p.rots[r])) return CKKS_ERR_NO_KEY;
        const size_t bp = (size_t)2 * level * c->N * sizeof(u64), need = ckks_cache_append_workspace_bytes(c, d, level, n);
        if (!ws || ws_bytes < need) return CKKS_ERR_WORKSPACE;
        Buffers buffers;
        for (const Side &sd : sides)
            for (uint32_t i = 0; i < n; i++) {
                const void *pg = sd.page[pages[i]].data, *o = sd.out[pages[i]].data;
                buffers.read(sd.in[i].data, (size_t)2 * sd.pitch * c->N * sizeof(u64));
                if (pg != o) buffers.read(pg, bp);
                buffers.write(o, bp);
            }
        if (rotated) read_factors(c, d, p, cosv, sinv, table_rows, keys, nkeys, buffers);
        buffers.write(ws, need);
        if (!buffers.apart()) return CKKS_ERR_ARG;
        DeviceGuard guard(c->device);
        std::vector<std::vector<Item>> items(sides.size());
        for (size_t x = 0; x < sides.size(); x++)
            for (uint32_t i = 0; i < n; i++)
                items[x].push_back(Item{(const u64 *)sides[x].in[i].data, (const u64 *)sides[x].page[pages[i]].data, (u64 *)sides[x].out[pages[i]].data, spans[i].row, spans[i].begin,
                                        spans[i].end});
        // pages that are filled whole need no mask: with any of them the values go on their own
        bool together = rotated && in_v;
        for (uint32_t i = 0; i < n; i++) together = together && (spans[i].begin || spans[i].end < d->token_inner);
        if (rotated)
            rotate_items(c, d, p, items[0], sides[0].pitch, level + 1, cosv, sinv, keys, nkeys, ws, (cudaStream_t)stream, together ? &items[1] : nullptr, together ? sides[1].pitch : 0);
        for (size_t x = rotated ? 1 : 0; x < sides.size() && !together; x++)
            append_items(c, d->token_inner, items[x], sides[x].pitch, level + 1, ws, (cudaStream_t)stream);
        rc = finish(c);
        for (const Side &sd : sides)
            for (uint32_t i = 0; i < n && rc == CKKS_OK; i++) {
                sd.out[pages[i]].scale = sd.page[pages[i]].scale;
                sd.out[pages[i]].level = level; sd.out[pages[i]].ncomp = 2;
            }
        return rc;
    });
}
