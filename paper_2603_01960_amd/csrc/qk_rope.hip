// C-ABI of the norm and rotation of queries and keys: validation and dispatch.  See include/tiled_sdpa.h.
#include "tiled_sdpa.h"

#include <cmath>
#include <cstdint>
#include <limits>

#include "qk_rope_kernel.h"

namespace {

int validate(const tsdpa_rope &p, bool cache, int pages, int block_rows)
{
    if (p.dtype != TSDPA_F16 && p.dtype != TSDPA_BF16) return TSDPA_ERR_BAD_DTYPE;
    if ((p.q_weight || p.k_weight) && p.weight_dtype != TSDPA_F32 && p.weight_dtype != p.dtype) return TSDPA_ERR_BAD_DTYPE;
    if (p.D != 64 && p.D != 96 && p.D != 128 && p.D != 160) return TSDPA_ERR_UNSUPPORTED_D;
    const int64_t most = std::numeric_limits<int>::max();
    if (p.B < 0 || p.S < 0 || p.H < 0 || p.Hkv < 0 || p.rot < 0 || p.rot > p.D || p.rot % 16 != 0 || (p.axes && p.n_axes < 1))
        return TSDPA_ERR_BAD_SHAPE;
    // rows of all heads of all tokens are counted in an int (products of three: two at a time)
    const int64_t heads = (int64_t)p.H + 2 * (int64_t)p.Hkv, tokens = (int64_t)p.B * p.S;
    if (heads > most / 2 || (tokens > 0 && heads > 0 && (heads + 64) > most / tokens) || tokens > most / 4) return TSDPA_ERR_BAD_SHAPE;
    if (cache && (pages < 0 || block_rows < 1 || (int64_t)pages * block_rows > most)) return TSDPA_ERR_BAD_SHAPE;
    return TSDPA_OK;
}

bool misaligned(const void *at, uintptr_t bytes) { return ((uintptr_t)at & (bytes - 1)) != 0; }

// A row's strides: what a 16-byte load needs, and (for rows that are written) no two of them in one place.
bool bad_strides(const tsdpa_rows &r, int B, int S, int heads, int D, bool written)
{
    struct Dim { long long stride; int size; } d[3] = {{r.batch, B}, {r.row, S}, {r.head, heads}};
    for (const Dim &x : d)
        if (x.size > 1 && (x.stride < 0 || (x.stride & 7) != 0)) return true;      // (one row has no stride)
    if (!written) return false;
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (d[j].stride > d[j + 1].stride) {
                const Dim x = d[j];
                d[j] = d[j + 1];
                d[j + 1] = x;
            }
    // (each dimension steps over all of the smaller ones; enough, and true of every view of a dense tensor)
    __int128 span = D;
    for (const Dim &x : d) {
        if (x.size <= 1) continue;
        if (x.stride < span) return true;
        span += (__int128)x.stride * (x.size - 1);
    }
    return false;
}

tsdpa::RopeRows rows(const tsdpa_rows *r) { return tsdpa::RopeRows{r->data, r->batch, r->row, r->head}; }

tsdpa::RopeArgs arguments(const tsdpa_rope &p, void *stream)
{
    tsdpa::RopeArgs a{};
    a.weight[0] = p.q_weight;
    a.weight[1] = p.k_weight;
    a.weight32 = p.weight_dtype == TSDPA_F32;
    a.positions = p.positions;
    a.pos_batch = p.pos_batch;
    a.pos_axis = p.axes ? p.pos_axis : 0;
    a.inv_freq = p.inv_freq;
    a.axes = p.axes;
    a.n_axes = p.axes ? p.n_axes : 1;
    a.B = p.B;
    a.S = p.S;
    a.heads[0] = p.H;
    a.heads[1] = a.heads[2] = p.Hkv;
    a.rot = p.rot;
    a.interleaved = (p.flags & TSDPA_FLAG_INTERLEAVED) ? 1 : 0;
    a.eps = p.eps;
    a.by_s = tsdpa::divisor((uint32_t)(p.S > 0 ? p.S : 1));
    a.stream = (hipStream_t)stream;
    return a;
}

// The checks that every call has, in the header's order, after those of its shape.
int check_common(const tsdpa_rope &p)
{
    if (p.rot > 0 && (!p.positions || !p.inv_freq)) return TSDPA_ERR_NULL_PTR;
    if (misaligned(p.q_weight, 16) || misaligned(p.k_weight, 16) || misaligned(p.positions, 4) || misaligned(p.inv_freq, 4) || misaligned(p.axes, 4))
        return TSDPA_ERR_MISALIGNED;
    return TSDPA_OK;
}

int forward(const tsdpa_rope *p, const tsdpa_rows *q, const tsdpa_rows *k, const tsdpa_rows *v, const int *slots, void *q_out, void *k_out,
            void *v_out, int pages, int block_rows, bool cache, void *stream)
{
    if (!p || !q || !k || (cache && !v)) return TSDPA_ERR_NULL_PTR;
    int st = validate(*p, cache, pages, block_rows);
    if (st != TSDPA_OK) return st;
    if ((int64_t)p->B * p->S == 0 || p->H + p->Hkv == 0) return TSDPA_OK;
    // (a cache without pages has no memory: every slot lies past its end)
    const bool stored = cache && pages > 0;
    if ((p->H > 0 && (!q->data || !q_out)) || (p->Hkv > 0 && (!k->data || (!cache && !k_out) || (cache && (!v->data || !slots)))) ||
        (p->Hkv > 0 && stored && (!k_out || !v_out)))
        return TSDPA_ERR_NULL_PTR;
    st = check_common(*p);
    if (st != TSDPA_OK) return st;
    if (misaligned(q->data, 16) || misaligned(k->data, 16) || (cache && misaligned(v->data, 16)) || misaligned(q_out, 16) || misaligned(k_out, 16) ||
        misaligned(v_out, 16) || misaligned(slots, 4))
        return TSDPA_ERR_MISALIGNED;
    if (bad_strides(*q, p->B, p->S, p->H, p->D, false) || bad_strides(*k, p->B, p->S, p->Hkv, p->D, false) ||
        (cache && bad_strides(*v, p->B, p->S, p->Hkv, p->D, false)))
        return TSDPA_ERR_BAD_STRIDE;
    if (!(p->eps >= 0.f) || std::isinf(p->eps)) return TSDPA_ERR_BAD_EPS;
    tsdpa::RopeArgs a = arguments(*p, stream);
    a.x[0] = rows(q);
    a.x[1] = rows(k);
    if (cache) a.x[2] = rows(v);
    a.out[0] = q_out;
    a.out[1] = k_out;
    a.out[2] = v_out;
    a.slots = slots;
    a.cache_rows = cache ? pages * block_rows : 0;
    a.block_rows = block_rows;
    a.by_rows = tsdpa::divisor((uint32_t)(cache ? block_rows : 1));
    const int err = p->dtype == TSDPA_F16 ? tsdpa::launch_rope_f16(p->D, cache, a) : tsdpa::launch_rope_bf16(p->D, cache, a);
    return err == 0 ? TSDPA_OK : TSDPA_ERR_LAUNCH;
}

}  // namespace

extern "C" {

int tiled_sdpa_qk_norm_rope(const tsdpa_rope *p, const tsdpa_rows *q, const tsdpa_rows *k, void *q_out, void *k_out, void *stream)
{
    return forward(p, q, k, nullptr, nullptr, q_out, k_out, nullptr, 0, 1, false, stream);
}

int tiled_sdpa_qk_norm_rope_cache(const tsdpa_rope *p, const tsdpa_rows *q, const tsdpa_rows *k, const tsdpa_rows *v, const int *slots,
                                  void *q_out, void *k_cache, void *v_cache, int pages, int block_rows, void *stream)
{
    return forward(p, q, k, v, slots, q_out, k_cache, v_cache, pages, block_rows, true, stream);
}

unsigned long long tiled_sdpa_qk_norm_rope_bwd_workspace_bytes(int B, int S, int D)
{
    if (B < 0 || S < 0 || D < 0) return 0;
    return (unsigned long long)tsdpa::kRopeBwdMost * D * sizeof(float);
}

int tiled_sdpa_qk_norm_rope_bwd(const tsdpa_rope *p, const void *dq_out, const void *dk_out, const tsdpa_rows *q, const tsdpa_rows *k,
                                const tsdpa_rows *dq, const tsdpa_rows *dk, void *dq_weight, void *dk_weight,
                                void *workspace, unsigned long long workspace_bytes, void *stream)
{
    if (!p || !q || !k || !dq || !dk) return TSDPA_ERR_NULL_PTR;
    int st = validate(*p, false, 0, 1);
    if (st != TSDPA_OK) return st;
    const bool norms = p->q_weight || p->k_weight;
    // (without rows the weights' gradients are still results: zeros)
    const bool empty = (int64_t)p->B * p->S == 0 || p->H + p->Hkv == 0;
    if (empty && !norms) return TSDPA_OK;
    if ((p->q_weight && !dq_weight) || (p->k_weight && !dk_weight)) return TSDPA_ERR_NULL_PTR;
    if (!empty && ((p->H > 0 && (!dq_out || !dq->data || (p->q_weight && !q->data))) ||
                   (p->Hkv > 0 && (!dk_out || !dk->data || (p->k_weight && !k->data)))))
        return TSDPA_ERR_NULL_PTR;
    if (!empty) {
        st = check_common(*p);
        if (st != TSDPA_OK) return st;
    }
    const uintptr_t size = p->weight_dtype == TSDPA_F32 ? 4 : 2;
    if (misaligned(dq_out, 16) || misaligned(dk_out, 16) || (p->q_weight && misaligned(q->data, 16)) || (p->k_weight && misaligned(k->data, 16)) ||
        misaligned(dq->data, 16) || misaligned(dk->data, 16) || (p->q_weight && misaligned(dq_weight, size)) ||
        (p->k_weight && misaligned(dk_weight, size)))
        return TSDPA_ERR_MISALIGNED;
    if ((p->q_weight && bad_strides(*q, p->B, p->S, p->H, p->D, false)) || (p->k_weight && bad_strides(*k, p->B, p->S, p->Hkv, p->D, false)) ||
        bad_strides(*dq, p->B, p->S, p->H, p->D, true) || bad_strides(*dk, p->B, p->S, p->Hkv, p->D, true))
        return TSDPA_ERR_BAD_STRIDE;
    if (!(p->eps >= 0.f) || std::isinf(p->eps)) return TSDPA_ERR_BAD_EPS;
    if (norms && (!workspace || misaligned(workspace, 16) || workspace_bytes < tiled_sdpa_qk_norm_rope_bwd_workspace_bytes(p->B, p->S, p->D)))
        return TSDPA_ERR_WORKSPACE;
    tsdpa::RopeArgs a = arguments(*p, stream);
    a.dy[0] = dq_out;
    a.dy[1] = dk_out;
    a.x[0] = rows(q);
    a.x[1] = rows(k);
    a.grad[0] = rows(dq);
    a.grad[1] = rows(dk);
    a.out[0] = p->q_weight ? dq_weight : nullptr;
    a.out[1] = p->k_weight ? dk_weight : nullptr;
    a.partial = (float *)workspace;
    const int err = p->dtype == TSDPA_F16 ? tsdpa::launch_rope_bwd_f16(p->D, a) : tsdpa::launch_rope_bwd_bf16(p->D, a);
    return err == 0 ? TSDPA_OK : TSDPA_ERR_LAUNCH;
}

}  // extern "C"
