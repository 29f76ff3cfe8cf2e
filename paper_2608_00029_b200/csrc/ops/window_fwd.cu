// Forward of the attention with a sliding window and sinks (include/nova_window.h).
//
// A work item is one 128-row query tile of one head; the keys in its reach go by in steps of 64: first those of the sinks that lie
// before the window, then the window's (key_span).  Items are short, a few steps up to a few dozen, so what lies between two of
// them counts: TWO CTAs share an SM, each with half of its tensor memory, and what one of them waits for, at an item's ends or in
// the chain products -> softmax -> product of a step, the other fills.  Within an item S runs a step ahead.
// (The form with one CTA and two softmax groups, by which attn_fwd.cu works on single tiles, took 34.7 us for a window of 256 and 4
// sinks at B=8, H=12, T=1024, D=64, longer than the whole triangle; this one takes 24.5 with O_rest, 22.6 without.)
//
//   S = Q K_s^T      (smem x smem -> one of two buffers in TMEM)
//   P = 2^(S c - m c) as bf16 over S (and what rounding takes from it beside it: launch_window_fwd), running maximum and sum in
//       registers, one thread per row
//   O += P V_s       (TMEM x smem); rescaled by the row's thread when its maximum has grown by more than 2^8
//
// What bounds it: a step's chain, some 1400 clocks in a softmax warp besides its waits (512 of them the exp2 unit) and as long again
// until the next S, against 512 clocks of the exp2 unit and 320 (D=64) or 640 (D=128) of the tensor pipe; 2900 clocks at an item's
// end.  At D=64 the tensor pipe is 17 % busy and the exp2 unit 28 % (the shape above, cold), at D=128 47 and 44 % (B=2, H=12 on 4,
// T=8192, window 1024: 110 us, 0.88 PFLOP/s of kept pairs; without any softmax 96).  Of a step's 64 keys a warp leaves out the half that
// none of its 32 rows keeps, at the diagonal and at the window's far end; a step of sinks takes products only as wide as there
// are sinks.
// O (and what rounding takes from it) goes straight from the registers to memory, 64 bytes of a row per thread at a time:
// there is no shared memory to stage it in, and no need to wait for it.
//
// 192 threads: warp 0 TMA producer, warp 1 UMMA issuer, warps 2-5 softmax.  Items are handed out dynamically (WorkRing).
#include <algorithm>
#include <type_traits>

#include "../api.h"
#include "../ptx.cuh"
#include "window.h"

namespace nova {
namespace {

constexpr int kThreads = 192;
constexpr int kTmemCols = 256;
constexpr int kStep = kKeyStep;
constexpr float kRescaleThreshold = 8.0f;  // log2 units
constexpr int kFewKeys = 64;  // that a row keeps, window and sinks (see launch_window_fwd)

template <int D>
struct Cfg {
    static constexpr int kHalves = D / kBoxCols;
    static constexpr int kHalfStepBytes = kStep * 128;  // one [64 keys x 64 bf16] box
    static constexpr int kStepBytes = kHalves * kHalfStepBytes;
    static constexpr int kTileBytes = kHalves * kHalfTileBytes;
    static constexpr int kQStages = D == 64 ? 2 : 1;
    static constexpr int kStages = D == 64 ? 4 : 2;  // of K, and of V
    static constexpr int kOffK = kQStages * kTileBytes;
    static constexpr int kOffV = kOffK + kStages * kStepBytes;
    static constexpr int kOffBar = kOffV + kStages * kStepBytes;
    static constexpr int kSmemBytes = kOffBar + 512 + 1024;
    static_assert(2 * (kSmemBytes + 1024) <= 233472, "two CTAs to an SM");
    static constexpr int kColS = 0, kColO = 2 * kStep;  // S: + 64 * buffer
};

struct Bars {
    uint64_t q_full[2], q_empty[2];
    uint64_t k_full[4], k_empty[4], v_full[4], v_empty[4];
    uint64_t s_full[2], p_ready[2];  // by buffer
    uint64_t pv_done, o_done;        // a P V has completed; the last one of an item has
    uint64_t drain;
    WorkRing ring;
    uint32_t tmem_base;
    int abort_flag;
};
static_assert(sizeof(Bars) <= 512, "barrier block");

struct Work {
    int BH, n_tiles, T, H;
    uint32_t orders;  // coordinate orders of the Q, K, V tensor maps, four bits each
    Window win;
    // the last rows first, as everywhere
    __device__ __forceinline__ void get(int idx, int* qt, int* bh, KeySpan* span) const {
        const int order = idx / BH;
        *qt = n_tiles - 1 - order;
        *bh = idx - order * BH;
        *span = key_span(win, *qt * kBlockQ, kBlockQ, T, kStep);
    }
    // Keys of step j that are looked at: a step of sinks ends with them.
    __device__ __forceinline__ int width(const KeySpan& span, int j) const {
        return j < span.sinks ? min(kStep, win.sinks - j * kStep) : kStep;
    }
};

template <int D, bool kStrided>
__device__ __forceinline__ void producer(const CUtensorMap* tmQ, const CUtensorMap* tmK, const CUtensorMap* tmV, uint8_t* smem,
                                         Bars* bars, const Work& wk) {
    using C = Cfg<D>;
    volatile int* abort_flag = &bars->abort_flag;
    bool ok = true, clc_pending = false;
    int w = 0, n_q = 0, n_k = 0, n_v = 0, st = 0;  // items; loads of Q, K, V requested; stage
    uint32_t ph = 0;
    int item = blockIdx.x;
    for (;;) {
        ok = bars->ring.publish(w, item, abort_flag, kWaitLimitCycles);
        if (!ok || item < 0) break;
        int qt, bh;
        KeySpan span;
        wk.get(item, &qt, &bh, &span);
        const int head = kStrided ? bh % wk.H : 0, batch = kStrided ? bh / wk.H : 0;
        const int kv_head = head / wk.win.group, kv_bh = bh / wk.win.group;
        const int qs = w % C::kQStages;
        ok = mbar_wait(&bars->q_empty[qs], ((w / C::kQStages) & 1) ^ 1, abort_flag);
        if (!ok) break;
        mbar_expect_tx(&bars->q_full[qs], C::kTileBytes);  // rows past T arrive as zeros
        ++n_q;
#pragma unroll
        for (int h = 0; h < C::kHalves; ++h)
            tma_load_tile<kStrided>(smem + qs * C::kTileBytes + h * kHalfTileBytes, tmQ, &bars->q_full[qs], wk.orders & 15,
                                    h * kBoxCols, qt * kBlockQ, head, batch, bh);
        for (int j = 0; j < span.n; ++j) {
            const int key0 = span.at(j) * kStep;
            ok = mbar_wait(&bars->k_empty[st], ph ^ 1, abort_flag);
            if (!ok) break;
            mbar_expect_tx(&bars->k_full[st], C::kStepBytes);
            ++n_k;
#pragma unroll
            for (int h = 0; h < C::kHalves; ++h)
                tma_load_tile<kStrided>(smem + C::kOffK + st * C::kStepBytes + h * C::kHalfStepBytes, tmK, &bars->k_full[st],
                                        (wk.orders >> 4) & 15, h * kBoxCols, key0, kv_head, batch, kv_bh);
            ok = mbar_wait(&bars->v_empty[st], ph ^ 1, abort_flag);
            if (!ok) break;
            mbar_expect_tx(&bars->v_full[st], C::kStepBytes);
            ++n_v;
#pragma unroll
            for (int h = 0; h < C::kHalves; ++h)
                tma_load_tile<kStrided>(smem + C::kOffV + st * C::kStepBytes + h * C::kHalfStepBytes, tmV, &bars->v_full[st],
                                        (wk.orders >> 8) & 15, h * kBoxCols, key0, kv_head, batch, kv_bh);
            if (++st == C::kStages) {
                st = 0;
                ph ^= 1;
            }
        }
        if (!ok) break;
        // all loads of this item are on their way: claim the next one now, and no earlier
        bars->ring.request();
        clc_pending = true;
        ok = bars->ring.answer(w, &item, abort_flag, kWaitLimitCycles);
        if (!ok) break;
        clc_pending = false;
        ++w;
    }
    if (!ok) {  // giving up: let what is in flight land before the CTA's shared memory goes away
        int none = 0;
        if (clc_pending) (void)mbar_wait(&bars->ring.answer_bar, w & 1, &none);
        for (int x = n_q > C::kQStages ? n_q - C::kQStages : 0; x < n_q; ++x)
            (void)mbar_wait(&bars->q_full[x % C::kQStages], (x / C::kQStages) & 1, &none);
        for (int x = n_k > C::kStages ? n_k - C::kStages : 0; x < n_k; ++x)
            (void)mbar_wait(&bars->k_full[x % C::kStages], (x / C::kStages) & 1, &none);
        for (int x = n_v > C::kStages ? n_v - C::kStages : 0; x < n_v; ++x)
            (void)mbar_wait(&bars->v_full[x % C::kStages], (x / C::kStages) & 1, &none);
    }
}

// UMMA issuer: the whole warp in uniform control flow, one elected lane issues.
template <int D, bool kSplit>
__device__ __forceinline__ void mma(uint8_t* smem, Bars* bars, uint32_t tmem_base, const Work& wk) {
    using C = Cfg<D>;
    volatile int* abort_flag = &bars->abort_flag;
    constexpr uint32_t kIdescPV = umma_idesc_bf16(128, D, 0, 1);
    const uint32_t hi = umma_desc_hi_sw128(1024);
    const uint32_t q_k0 = umma_desc_lo(smem_u32(smem), 16), k_k0 = umma_desc_lo(smem_u32(smem + C::kOffK), 16);
    const uint32_t v_m0 = umma_desc_lo(smem_u32(smem + C::kOffV), C::kHalfStepBytes);
    const bool el = elect_one();
    const int lane = threadIdx.x & 31;
    bool ok = true;
    int w = 0, g = 0;  // items, steps of all items whose P V has been issued
    int st_k = 0, st_v = 0;
    uint32_t ph_k = 0, ph_v = 0;
    int gk = 0;  // steps of all items whose Q K^T has been issued
    // S of the next step into buffer gk & 1, whose last P was consumed by a P V queued earlier.
    auto issue_qk = [&](int qs, int width, bool last) {
        ok = mbar_wait(&bars->k_full[st_k], ph_k, abort_flag);
        if (!ok) return;
        tc_fence_after();
        if (el) {
            const uint32_t idesc = umma_idesc_bf16(128, (width + 15) / 16 * 16, 0, 0);
            const uint32_t q = q_k0 + qs * (C::kTileBytes >> 4), b = k_k0 + st_k * (C::kStepBytes >> 4);
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
                umma_ss(tmem_base + C::kColS + kStep * (gk & 1),
                        umma_desc_join(q + (((k / 4) * kHalfTileBytes + (k % 4) * 32) >> 4), hi),
                        umma_desc_join(b + (((k / 4) * C::kHalfStepBytes + (k % 4) * 32) >> 4), hi), idesc, k > 0 ? 1u : 0u);
            tc_commit(&bars->s_full[gk & 1]);
            tc_commit(&bars->k_empty[st_k]);
            if (last) tc_commit(&bars->q_empty[qs]);
        }
        __syncwarp();
        ++gk;
        if (++st_k == C::kStages) {
            st_k = 0;
            ph_k ^= 1;
        }
    };
    constexpr int kNotPeeked = -3;
    int peeked = kNotPeeked;  // the next item's number, if it was looked at from inside the current item
    int ahead = 0;            // ... and how many of its Q K^T were queued from there
    for (;;) {
        const int item = (peeked != kNotPeeked) ? peeked : bars->ring.take(w, lane, abort_flag, kWaitLimitCycles);
        peeked = kNotPeeked;
        if (item < 0) {
            ok = (item == -1);
            break;
        }
        int qt, bh;
        KeySpan span;
        wk.get(item, &qt, &bh, &span);
        const int n = span.n, qs = w % C::kQStages;
        if (ahead == 0) {
            ok = mbar_wait(&bars->q_full[qs], (w / C::kQStages) & 1, abort_flag);
            if (ok) issue_qk(qs, wk.width(span, 0), n == 1);
        }
        ahead = 0;
        if (ok && n > 1) issue_qk(qs, wk.width(span, 1), n == 2);
        for (int j = 0; j < n && ok; ++j, ++g) {
            if (j + 1 == n && bars->ring.published(w + 1)) {
                // Last step: S of the next item's first, if its Q and K have landed, so that the softmax warps find it there.
                peeked = bars->ring.take(w + 1, lane, abort_flag, kWaitLimitCycles);
                if (peeked >= 0) {
                    const int qs2 = (w + 1) % C::kQStages;
                    const bool there = mbar_test(&bars->q_full[qs2], ((w + 1) / C::kQStages) & 1) && mbar_test(&bars->k_full[st_k], ph_k);
                    if (__all_sync(0xffffffffu, there)) {
                        int qt2, bh2;
                        KeySpan span2;
                        wk.get(peeked, &qt2, &bh2, &span2);
                        issue_qk(qs2, wk.width(span2, 0), span2.n == 1);
                        ahead = 1;
                    }
                }
            }
            if (ok) ok = mbar_wait(&bars->v_full[st_v], ph_v, abort_flag);
            if (ok) ok = mbar_wait(&bars->p_ready[g & 1], (g >> 1) & 1, abort_flag);
            if (!ok) break;
            tc_fence_after();
            // O += P V: P from TMEM (16 keys = 8 packed columns per instruction), V MN-major (rows = keys, 64 head-dim elements
            // per 128-byte row).  The softmax warps have read the previous item's O before they made this item's first P.
            if (el) {
                const int chunks = (wk.width(span, j) + 15) / 16;
                const uint32_t p = tmem_base + C::kColS + kStep * (g & 1), v = v_m0 + st_v * (C::kStepBytes >> 4);
#pragma unroll
                for (int k = 0; k < kStep / 16; ++k) {
                    if (k < chunks) {
                        umma_ts(tmem_base + C::kColO, p + k * 8, umma_desc_join(v + k * 128, hi), kIdescPV, (j > 0 || k > 0) ? 1u : 0u);
                        if (kSplit) umma_ts(tmem_base + C::kColO, p + 32 + k * 8, umma_desc_join(v + k * 128, hi), kIdescPV, 1u);
                    }
                }
                tc_commit(&bars->pv_done);
                tc_commit(&bars->v_empty[st_v]);
                if (j + 1 == n) tc_commit(&bars->o_done);
            }
            __syncwarp();
            if (++st_v == C::kStages) {
                st_v = 0;
                ph_v ^= 1;
            }
            if (j + 2 < n) issue_qk(qs, wk.width(span, j + 2), j + 3 == n);
        }
        if (!ok) break;
        ++w;
    }
    if (!ok) {  // drain whatever was issued before leaving so TMEM can be released safely
        int none = 0;
        if (el) tc_commit(&bars->drain);
        __syncwarp();
        (void)mbar_wait(&bars->drain, 0, &none);
    }
}

// What rounding took from two numbers, rounded in its turn.
__device__ __forceinline__ uint32_t rest_of(uint32_t packed, float x, float y) {
    return pack_bf16x2(x - __uint_as_float(packed << 16), y - __uint_as_float(packed & 0xffff0000u));
}

// 32 bytes: one access where the row is aligned to them.
__device__ __forceinline__ void store_32(uint16_t* p, const uint32_t* v, bool aligned) {
    if (aligned) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
                     "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                     : "memory");
    } else {
        *reinterpret_cast<uint4*>(p) = make_uint4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<uint4*>(p + 8) = make_uint4(v[4], v[5], v[6], v[7]);
    }
}

template <int D, bool kSplit>
__device__ __forceinline__ void softmax(Bars* bars, uint32_t tmem_base, uint16_t* __restrict__ O, uint16_t* __restrict__ rest,
                                        float* __restrict__ LSE, const TensorStrides& so, bool aligned, float scale, const Work& wk,
                                        int swarp, int lane) {
    using C = Cfg<D>;
    volatile int* abort_flag = &bars->abort_flag;
    const uint32_t lane_base = 32u * swarp;
    const uint32_t t_o = tmem_addr(tmem_base, lane_base, C::kColO);
    const float c = scale * kLog2e;
    const uint64_t c2 = f32x2_pack(c, c);
    const int T = wk.T;
    bool ok = true;
    int g = 0;  // steps of all items
    int item = bars->ring.take(0, lane, abort_flag, kWaitLimitCycles);
    for (int w = 0; item >= 0; ++w) {
        int qt, bh;
        KeySpan span;
        wk.get(item, &qt, &bh, &span);
        const int row0 = qt * kBlockQ + lane_base, row = row0 + lane;  // the warp's first row, the thread's
        const int last = min(row0 + 31, T - 1), kept_row = min(row, T - 1);
        float m_ref = -INFINITY, l = 0.f;  // -inf while there has been no key that the row keeps
        // Halves of 32 keys: does any of the warp's rows keep any of it, and all of them all of it?  The same in every lane.  (Found out
        // for a step while the P of the one before is on its way.)
        int key0;
        bool need[2], whole[2];
        auto look = [&](int j) {
            key0 = span.at(j) * kStep;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k0 = key0 + 32 * h;
                need[h] = k0 <= last && (k0 + 31 > row0 - wk.win.window || k0 < wk.win.sinks);
                whole[h] = k0 + 31 <= row0 && (k0 > row0 + 31 - wk.win.window || k0 + 31 < wk.win.sinks);
            }
        };
        look(0);
        for (int j = 0; j < span.n; ++j, ++g) {
            const int buf = g & 1;
            const uint32_t t_s = tmem_addr(tmem_base, lane_base, C::kColS + kStep * buf);
            ok = mbar_wait(&bars->s_full[buf], (g >> 1) & 1, abort_flag);
            if (!ok) break;
            tc_fence_after();
            uint32_t sr[kStep];
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (need[h]) tmem_ld_x32(t_s + 32 * h, sr + 32 * h);
            tmem_wait_ld();
            float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (!need[h]) continue;
                if (!whole[h]) {
                    const uint32_t kept = kept_keys_32(wk.win, kept_row, key0 + 32 * h);
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (!(kept >> i & 1u)) sr[32 * h + i] = 0xff800000u;  // -inf
                }
#pragma unroll
                for (int i = 0; i < 32; i += 2)
                    mx[i / 2 % 4] = fmax3(mx[i / 2 % 4], __uint_as_float(sr[32 * h + i]), __uint_as_float(sr[32 * h + i + 1]));
            }
            const float m_new = fmaxf(m_ref, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])));
            if (j == 0) {
                m_ref = m_new;
            } else if (__any_sync(0xffffffffu, (m_new - m_ref) * c > kRescaleThreshold)) {  // (-inf against -inf: no)
                const float f = m_new > m_ref ? ex2_approx((m_ref - m_new) * c) : 1.f;  // 0 from -inf
                m_ref = m_new;
                l *= f;
                // (that of step g - 2 has completed: S of this step, which is here, was issued after it)
                ok = mbar_wait(&bars->pv_done, (g - 1) & 1, abort_flag);
                if (!ok) break;
                tc_fence_after();
#pragma unroll 1
                for (int cb = 0; cb < D; cb += 16) {
                    uint32_t o[16];
                    tmem_ld_x16(t_o + cb, o);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                    tmem_st_x16(t_o + cb, o);
                }
            }
            // P = 2^(s * c - m * c).  Where the rounding of m * c is as large as the exponent's range (scores of the type's lowest
            // value) it is rounded up, which keeps P <= 1.
            const float mc_near = m_ref * c, mc_up = __fmul_ru(m_ref, c);
            const float mc = m_ref == -INFINITY ? 0.f : fabsf(mc_near) > 1e9f ? mc_up : mc_near;
            const uint64_t nmc2 = f32x2_pack(-mc, -mc);
            uint64_t acc[4] = {0, 0, 0, 0};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t pk[16], lo[kSplit ? 16 : 1];
                if (need[h]) {
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        const uint32_t* s = sr + 32 * h + i;
                        float x0, x1, x2, x3;
                        f32x2_unpack(f32x2_fma(f32x2_pack(__uint_as_float(s[0]), __uint_as_float(s[1])), c2, nmc2), x0, x1);
                        f32x2_unpack(f32x2_fma(f32x2_pack(__uint_as_float(s[2]), __uint_as_float(s[3])), c2, nmc2), x2, x3);
                        const float p0 = ex2_approx(x0), p1 = ex2_approx(x1), p2 = ex2_approx(x2), p3 = ex2_approx(x3);
                        acc[i / 2 % 4] = f32x2_add(acc[i / 2 % 4], f32x2_pack(p0, p1));
                        acc[i / 2 % 4 + 1] = f32x2_add(acc[i / 2 % 4 + 1], f32x2_pack(p2, p3));
                        pk[i / 2] = pack_bf16x2(p0, p1);
                        pk[i / 2 + 1] = pack_bf16x2(p2, p3);
                        if constexpr (kSplit) {
                            lo[i / 2] = rest_of(pk[i / 2], p0, p1);
                            lo[i / 2 + 1] = rest_of(pk[i / 2 + 1], p2, p3);
                        }
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) pk[i] = lo[kSplit ? i : 0] = 0u;
                }
                tmem_st_x16(t_s + 16 * h, pk);
                if constexpr (kSplit) tmem_st_x16(t_s + 32 + 16 * h, lo);
            }
            float a0, a1, a2, a3;
            f32x2_unpack(f32x2_add(acc[0], acc[2]), a0, a1);
            f32x2_unpack(f32x2_add(acc[1], acc[3]), a2, a3);
            l += (a0 + a1) + (a2 + a3);
            look(j + 1);  // (past the last step it says nothing)
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->p_ready[buf]);
        }
        if (!ok) return;
        // ---- end of the item: what needs no O first, then O
        item = bars->ring.take(w + 1, lane, abort_flag, kWaitLimitCycles);
        const float inv_l = 1.0f / l;
        const long long b = bh / wk.H, at = b * so.b + (bh - b * wk.H) * so.h + row * so.t;
        if (row < T) LSE[static_cast<size_t>(bh) * T + row] = m_ref * scale + logf(l);
        // (Not pv_done: P V of the step before the last may be outstanding still, and a wait two phases on would pass at once.)
        ok = mbar_wait(&bars->o_done, w & 1, abort_flag);
        if (!ok) return;
        tc_fence_after();
#pragma unroll
        for (int cb = 0; cb < D; cb += 32) {
            uint32_t a[32], v[16], r[16];
            tmem_ld_x32(t_o + cb, a);
            tmem_wait_ld();
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                const float o0 = __uint_as_float(a[2 * x]) * inv_l, o1 = __uint_as_float(a[2 * x + 1]) * inv_l;
                v[x] = pack_bf16x2(o0, o1);
                r[x] = rest_of(v[x], o0, o1);
            }
            if (row < T) {
                store_32(O + at + cb, v, aligned);
                store_32(O + at + cb + 16, v + 8, aligned);
                if (rest != nullptr) {
                    store_32(rest + at + cb, r, aligned);
                    store_32(rest + at + cb + 16, r + 8, aligned);
                }
            }
            __syncwarp();
        }
        tc_fence_before();
    }
}

template <int D, bool kStrided, bool kSplit>
__global__ void __launch_bounds__(kThreads, 2)
window_fwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                  uint16_t* __restrict__ O, uint16_t* __restrict__ rest, float* __restrict__ LSE, const TensorStrides so,
                  bool aligned, const Work wk, float scale, int* __restrict__ dev_status) {
    using C = Cfg<D>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    Bars* bars = reinterpret_cast<Bars*>(smem + C::kOffBar);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < 2; ++s) {
            mbar_init(&bars->q_full[s], 1);
            mbar_init(&bars->q_empty[s], 1);
            mbar_init(&bars->s_full[s], 1);
            mbar_init(&bars->p_ready[s], 4);
        }
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(&bars->k_full[s], 1);
            mbar_init(&bars->k_empty[s], 1);
            mbar_init(&bars->v_full[s], 1);
            mbar_init(&bars->v_empty[s], 1);
        }
        mbar_init(&bars->pv_done, 1);
        mbar_init(&bars->o_done, 1);
        mbar_init(&bars->drain, 1);
        bars->ring.init(1 + 4);  // issuer, softmax warps
        bars->abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&tmQ);
        tma_prefetch_desc(&tmK);
        tma_prefetch_desc(&tmV);
    }
    if (warp == 1) {
        tmem_alloc(&bars->tmem_base, kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = bars->tmem_base;
    griddep_launch_dependents();
    griddep_wait();

    if (warp == 0) {
        if (lane == 0) producer<D, kStrided>(&tmQ, &tmK, &tmV, smem, bars, wk);
    } else if (warp == 1) {
        mma<D, kSplit>(smem, bars, tmem_base, wk);
    } else {
        softmax<D, kSplit>(bars, tmem_base, O, rest, LSE, so, aligned, scale, wk, warp & 3, lane);
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem_base, kTmemCols);
    if (threadIdx.x == 0 && bars->abort_flag != 0) atomicExch(dev_status, kDevTimeout);
}

// Calls f with the kernel that is meant and its shared memory.
template <typename F>
cudaError_t with_kernel(int D, bool strided, bool split, F&& f) {
    auto of = [&](auto d, auto st) {
        constexpr int kD = decltype(d)::value;
        constexpr bool kStrided = decltype(st)::value;
        return split ? f(window_fwd_kernel<kD, kStrided, true>, Cfg<kD>::kSmemBytes) : f(window_fwd_kernel<kD, kStrided, false>, Cfg<kD>::kSmemBytes);
    };
    auto with_d = [&](auto d) { return strided ? of(d, std::true_type{}) : of(d, std::false_type{}); };
    return D == 64 ? with_d(std::integral_constant<int, 64>{}) : with_d(std::integral_constant<int, 128>{});
}

}  // namespace

cudaError_t configure_window_fwd() {
    cudaError_t e = cudaSuccess;
    for (int k = 0; k < 8 && e == cudaSuccess; ++k)
        e = with_kernel(k & 1 ? 64 : 128, (k & 2) != 0, (k & 4) != 0, [](auto kernel, int smem) {
            return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        });
    return e;
}

cudaError_t launch_window_fwd(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, bool strided, uint32_t orders,
                              __nv_bfloat16* O, __nv_bfloat16* rest, float* LSE, const TensorStrides& so, const AttnShape& s,
                              const Window& win, int* dev_status, cudaStream_t stream) {
    const int BH = s.B * s.H, n_tiles = (s.T + kBlockQ - 1) / kBlockQ;
    const dim3 grid(static_cast<unsigned>(n_tiles) * BH);  // one CTA per item; those that do not start at once are taken over
    const bool aligned = ((so.b | so.h | so.t) & 15) == 0 && ((reinterpret_cast<uintptr_t>(O) | reinterpret_cast<uintptr_t>(rest)) & 31) == 0;
    const Work wk{BH, n_tiles, s.T, s.H, orders, win};
    // Few keys to a row: the roundings of their weights do not average out in O, and reach dQ and dK through Delta.  Where O_rest is asked
    // for, the weights go into the product as two bf16 numbers then.  Error of dQ and dK over that of rounding the outputs alone, with
    // one number and with two: 1.46, 1.41 at 16 keys a row, 1.44, 1.42 at 128.  Time, with two and with one: B=8, H=12, T=1024, D=64,
    // window 64: 21.0, 19.3 us; a training pass of two heads, T=64, 18.1, 16.2 (more code to fetch).
    const bool split = rest != nullptr && std::min<long long>(static_cast<long long>(win.window) + win.sinks, s.T) <= kFewKeys;
    return with_kernel(s.D, strided, split, [&](auto kernel, int smem) {
        return launch_overlapped(kernel, grid, dim3(kThreads), smem, stream, tmQ, tmK, tmV, reinterpret_cast<uint16_t*>(O),
                                 reinterpret_cast<uint16_t*>(rest), LSE, so, aligned, wk, s.scale, dev_status);
    });
}

}  // namespace nova
