// C entry points of the decoder's operators: cross attention, its gradients, sampling.
#include <math.h>

#include "attend_launch.hpp"
#include "entry.hpp"
#include "sample.hpp"

using namespace tl;

namespace {

bool check_rows(const tl_rows &t, int dtype, long long rows, long long heads, int D, bool out)
{
    if (rows == 0) return true;
    if (!t.p || ((uintptr_t)t.p & (element_size(dtype) - 1)) || t.row < 0 || t.head < 0) return false;
    if (!out) return true;
    // rows of heads or heads of rows: the smaller stride spans D elements, the larger one everything the smaller one walks
    const bool by_row = heads == 1 || (rows > 1 && t.row >= t.head);
    const long long in_n = by_row ? heads : rows, in_s = by_row ? t.head : t.row, out_n = by_row ? rows : heads, out_s = by_row ? t.row : t.head;
    if (in_n > 1 && in_s < D) return false;
    return out_n <= 1 || out_s >= (in_n > 1 ? (in_n - 1) * in_s : 0) + D;
}

bool in_pieces(const tl_rows &t, int dtype, int D, int bytes)
{
    const int n = bytes / element_size(dtype);
    return D % n == 0 && t.row % n == 0 && t.head % n == 0 && ((uintptr_t)t.p & (bytes - 1)) == 0;
}

constexpr float LOG2_E = 1.4426950408889634f;    // exponentials are powers of two

// The kernels count in 32 bits and look up to 2^15 rows beyond the last one (4096 mask bytes at a time; 256 parts of whole stages) before they bound it.
constexpr int MOST_ROWS = INT32_MAX - 65536;

bool check(const tl_attention *a)
{
    if (!a || a->dtype < TL_DT_F32 || a->dtype > TL_DT_F16) return false;
    if (a->n_trees < 0 || a->n_q < 0 || a->n_kv < 0 || a->n_q > MOST_ROWS || a->n_kv > MOST_ROWS || a->n_heads < 1 || a->n_heads > 4096 || a->n_kv_heads < 1) return false;
    if (a->n_heads % a->n_kv_heads || a->head_dim < 1 || a->head_dim > 256) return false;
    if (!(a->scale > 0.f) || !isfinite(a->scale * LOG2_E)) return false;
    if (a->n_trees == 0) return a->n_q == 0 && a->n_kv == 0;
    if (!a->q_off || !a->kv_off) return false;
    return check_rows(a->q, a->dtype, a->n_q, a->n_heads, a->head_dim, false) && check_rows(a->k, a->dtype, a->n_kv, a->n_kv_heads, a->head_dim, false) &&
           check_rows(a->v, a->dtype, a->n_kv, a->n_kv_heads, a->head_dim, false);
}

// Parts that a loop of `stages` (on average) is cut into where its `blocks` workgroups do not fill the chip twice, as long as a part keeps two.
int splits(long long blocks, long long stages)
{
    const long long wanted = 2ll * compute_units();
    if (blocks >= wanted || stages < 4) return 1;
    const long long s = wanted / blocks < stages / 2 ? wanted / blocks : stages / 2;
    return (int)(s < 1 ? 1 : s > 256 ? 256 : s);
}

// Lists that mostly end within a stage need no second one in LDS, and twice as many workgroups then fit a compute unit.  Measured (us, two stages / one):
// 256 trees of 54 nodes, 33 rows each: bf16 x 64 read 23.9 / 20.0, fp32 x 64 58 / 50.
bool one_stage(long long rows, long long trees, int stage) { return 2 * rows <= 3ll * stage * trees; }

// Which form a forward takes, by the packed rows of a tree on average: the host does not know the lengths, and a batch with one tree much longer than the others
// waits for it (256 trees of 54 nodes, bf16 x 64, one token: 9 us; one of them of 20 000 nodes: 184).  Measured (us, 4 waves along the rows / 2 / 1): 256 trees of 9 to 99 nodes,
// 33 rows each, bf16 x 64: - / 24 / 38; fp32 x 64: - / 57 / 70; 64 trees of 2047 nodes half of them masked, 72 rows, fp32 x 64: 158 / 98 /
// 117; 8 trees of 3500 nodes, 3000 rows, bf16 x 128: 250 / 310 / -.  A single token's few rows want every wave on nodes of its own.
// Where row tiles do not fill the chip twice, a tree's nodes are divided among workgroups too, as long as a part keeps two stages.
// False where a launch would be too large.
bool plan(const tl_attention *a, AttPlan *out)
{
    AttPlan &p = *out;
    const long long rows = (long long)a->n_q * (a->n_heads / a->n_kv_heads);
    const int dp = att_padded(a->head_dim), size = element_size(a->dtype);
    p.wm = rows <= 16ll * a->n_trees && dp * size <= 512 ? 1 : rows <= 128ll * a->n_trees ? 2 : 4;
    p.bm = 32 * p.wm;
    p.bn = p.wm == 1 ? 128 : p.wm == 2 ? 64 : dp * size <= 256 ? 64 : 32;
    const long long slots = rows / p.bm + a->n_trees;
    if (slots > ATT_MOST_BLOCKS) return false;
    p.slots = (int)slots;
    p.splits = splits(slots * a->n_kv_heads, a->n_kv / ((long long)p.bn * a->n_trees));
    p.bufs = one_stage(a->n_kv, a->n_trees, p.bn) ? 1 : 2;
    return slots * p.splits * a->n_kv_heads <= ATT_MOST_BLOCKS && (p.splits == 1 || (long long)a->n_q * a->n_heads <= ATT_MOST_BLOCKS);
}

// The same for a backward pass, whose gradient of the queries sums over nodes and whose gradients of keys and values over rows.  Short trees (their rows,
// or their nodes, on average): fewer of them at a time, and the other side divided among the waves instead.  Measured (us, 2 / 4 waves side by
// side, each gradient launched by itself): 256 trees of 33 rows, 54 nodes, fp32 x 64: dQ 73 / 93, dK and dV 97 / 96; 25 such trees, x 30: 12 / 14 and 10 / 12; 8 trees
// of 1536 rows, 1200 nodes, bf16 x 128: 177 / 127 and 206 / 180.
bool back_plan(const tl_attention *a, AttBackPlan *out)
{
    AttBackPlan &p = *out;
    const long long rows = (long long)a->n_q * (a->n_heads / a->n_kv_heads), trees = a->n_trees, heads = a->n_kv_heads;
    p.q_waves = rows <= 128 * trees ? 2 : 4;
    p.kv_waves = a->n_kv <= 128 * trees ? 2 : 4;
    p.q_splits = a->n_q == 0 ? 1 : splits((rows / (32 * p.q_waves) + trees) * heads, a->n_kv / (64 * trees));
    p.kv_splits = a->n_kv == 0 ? 1 : splits((a->n_kv / (32 * p.kv_waves) + trees) * heads, rows / (64 * trees));
    p.q_bufs = one_stage(a->n_kv, trees, 64) ? 1 : 2;
    p.kv_bufs = one_stage(rows, trees, 64) ? 1 : 2;
    const int dp = att_padded(a->head_dim);
    const long long q_slots = rows / att_dq_rows(dp, p.q_waves) + trees, kv_slots = a->n_kv / att_dkv_nodes(dp, element_size(a->dtype), p.kv_waves) + trees;
    const long long row_heads = (long long)a->n_q * a->n_heads;
    const long long q_blocks = a->n_q > 0 ? q_slots * p.q_splits * heads : 0;
    // (a multiple of eight, so that consecutive workgroups of both kinds lie in one L2 domain)
    const long long kv_blocks = a->n_kv > 0 ? (kv_slots * p.kv_splits * heads + 7) & ~7ll : 0;
    const long long prepare = (row_heads + 15) / 16 + (a->kv_mask ? trees : 0);
    const long long sum_q = p.q_splits > 1 ? (row_heads + ATT_WAVES - 1) / ATT_WAVES : 0;
    const long long sum_kv = p.kv_splits > 1 ? (2ll * a->n_kv * heads + ATT_WAVES - 1) / ATT_WAVES : 0;
    if (q_slots > INT32_MAX || kv_slots > INT32_MAX || q_blocks + kv_blocks > ATT_MOST_BLOCKS || prepare > ATT_MOST_BLOCKS || sum_q + sum_kv > ATT_MOST_BLOCKS)
        return false;
    p.q_slots = (int)q_slots;
    p.kv_slots = (int)kv_slots;
    p.q_blocks = (int)q_blocks;
    p.kv_blocks = (int)kv_blocks;
    p.prepare_blocks = (int)prepare;
    p.sum_blocks_q = (int)sum_q;
    p.sum_blocks_kv = (int)sum_kv;
    return true;
}

long long workspace(const tl_attention *a, const AttPlan &p)
{
    const long long rh = (long long)a->n_q * a->n_heads;
    return p.splits > 1 ? round16(p.splits * rh * 4) + round16(p.splits * rh * a->head_dim * 4) : 0;
}

// The backward pass's workspace, in this order; null where a part is not needed.  Returns its size.
long long lay_out(const tl_attention *a, const AttBackPlan &p, char *base, AttArgs *x)
{
    long long at = 0;
    auto take = [&](long long bytes) {
        char *q = base + at;
        at += round16(bytes);
        return bytes ? (void *)q : nullptr;
    };
    const long long rh = (long long)a->n_q * a->n_heads, D = a->head_dim;
    x->delta = static_cast<float *>(take(rh * 4));
    x->ref = static_cast<float *>(take(rh * 4));
    x->size = static_cast<float *>(take(a->dtype == TL_DT_F16 ? rh * 4 : 0));
    x->list = static_cast<int32_t *>(take(a->kv_mask ? 4ll * a->n_kv : 0));
    x->live = static_cast<int32_t *>(take(a->kv_mask ? 4ll * a->n_trees : 0));
    x->part_q = static_cast<float *>(take(p.q_splits > 1 ? p.q_splits * rh * D * 4 : 0));
    x->part_kv = static_cast<float *>(take(p.kv_splits > 1 ? 2ll * p.kv_splits * a->n_kv * a->n_kv_heads * D * 4 : 0));
    return at;
}

AttArgs arguments(const tl_attention *a)
{
    AttArgs x = {};
    auto t = [](const tl_rows &r) { return AttTensor{r.p, r.row, r.head}; };
    x.q = t(a->q);
    x.k = t(a->k);
    x.v = t(a->v);
    x.q_off = a->q_off;
    x.kv_off = a->kv_off;
    x.mask = a->kv_mask;
    x.scale = a->scale;
    x.scale_log2 = a->scale * LOG2_E;
    x.n_trees = a->n_trees;
    x.n_q = a->n_q;
    x.n_kv = a->n_kv;
    x.Hq = a->n_heads;
    x.Hk = a->n_kv_heads;
    x.G = a->n_heads / a->n_kv_heads;
    x.D = a->head_dim;
    x.splits = 1;
    auto close = [&](const tl_rows &r) { return r.row < (1 << 20) && r.head < (1 << 20); };
    x.near = close(a->q) && close(a->k) && close(a->v);
    x.vec = in_pieces(a->q, a->dtype, a->head_dim, 16) && in_pieces(a->k, a->dtype, a->head_dim, 16) && in_pieces(a->v, a->dtype, a->head_dim, 16);
    return x;
}

bool pieces_of_4(const tl_rows &t, int dtype, int D) { return in_pieces(t, dtype, D, 4 * element_size(dtype)); }

// A workgroup a row; a launch has fewer than 2^32 threads in all, so very many rows take several.
template <typename T> hipError_t sample(SampleArgs a, int n_rows, hipStream_t st)
{
    constexpr int MOST = 1 << 21;
    hipError_t e = att_allow<k_sample<T>>(sizeof(SmpShared));
    while (e == hipSuccess) {
        const int n = n_rows < MOST ? n_rows : MOST;
        hipLaunchKernelGGL(k_sample<T>, dim3(n), dim3(SMP_THREADS), sizeof(SmpShared), st, a);
        e = hipGetLastError();
        n_rows -= n;
        if (n_rows == 0) break;
        a.logits = static_cast<const T *>(a.logits) + n * a.row;
        a.u += n;
        a.token += n;
        for (const float **x : {&a.temperature, &a.top_p, &a.min_p})
            if (*x) *x += n;
        if (a.top_k) a.top_k += n;
        if (a.logprob) a.logprob += n;
        if (a.kept) a.kept += n;
    }
    return e;
}

}  // namespace

extern "C" {

int tl_attend_workspace(const tl_attention *a, int backward, int64_t *bytes)
{
    if (!bytes || !check(a)) return TL_EINVAL;
    *bytes = 0;
    if (a->n_trees == 0) return TL_OK;
    if (backward) {
        AttBackPlan p;
        AttArgs unused;
        if (!back_plan(a, &p)) return TL_EINVAL;
        *bytes = lay_out(a, p, nullptr, &unused);
    } else if (a->n_q > 0) {
        AttPlan p;
        if (!plan(a, &p)) return TL_EINVAL;
        *bytes = workspace(a, p);
    }
    return TL_OK;
}

int tl_attend(const tl_attention *a, const tl_rows *o, float *lse, void *workspace_p, int64_t workspace_bytes, void *hip_stream)
{
    if (!check(a) || !o || !check_rows(*o, a->dtype, a->n_q, a->n_heads, a->head_dim, true)) return TL_EINVAL;
    if (a->n_trees == 0 || a->n_q == 0) return TL_OK;
    AttPlan p;
    if (!plan(a, &p)) return TL_EINVAL;
    const long long need = workspace(a, p);
    if (need > workspace_bytes) return TL_ELIMIT;
    if (need > 0 && (!workspace_p || ((uintptr_t)workspace_p & 15))) return TL_EINVAL;
    AttArgs x = arguments(a);
    x.o = AttTensor{o->p, o->row, o->head};
    x.lse = lse;
    x.vec_out = pieces_of_4(*o, a->dtype, a->head_dim);
    x.slots = p.slots;
    x.splits = p.splits;
    x.bufs = p.bufs;
    if (p.splits > 1) {
        x.part_lse = static_cast<float *>(workspace_p);
        x.part_o = reinterpret_cast<float *>(static_cast<char *>(workspace_p) + round16((long long)p.splits * a->n_q * a->n_heads * 4));
    }
    const hipStream_t st = (hipStream_t)hip_stream;
    const hipError_t e = a->dtype == TL_DT_F32 ? attend_forward<float>(x, p, st) : a->dtype == TL_DT_BF16 ? attend_forward<bf16_t>(x, p, st) : attend_forward<f16_t>(x, p, st);
    return e == hipSuccess ? TL_OK : TL_EHIP;
}

int tl_attend_backward(const tl_attention *a, const tl_rows *o, const float *lse, const tl_rows *d_o, const tl_rows *d_q, const tl_rows *d_k,
                       const tl_rows *d_v, void *workspace_p, int64_t workspace_bytes, void *hip_stream)
{
    if (!check(a) || !o || !d_o || !d_q || !d_k || !d_v) return TL_EINVAL;
    const int dt = a->dtype, D = a->head_dim;
    if (!check_rows(*o, dt, a->n_q, a->n_heads, D, false) || !check_rows(*d_o, dt, a->n_q, a->n_heads, D, false) ||
        !check_rows(*d_q, dt, a->n_q, a->n_heads, D, true) || !check_rows(*d_k, dt, a->n_kv, a->n_kv_heads, D, true) ||
        !check_rows(*d_v, dt, a->n_kv, a->n_kv_heads, D, true))
        return TL_EINVAL;
    if (a->n_trees == 0) return TL_OK;
    AttBackPlan p;
    if (!back_plan(a, &p)) return TL_EINVAL;
    AttArgs x = arguments(a);
    const long long need = lay_out(a, p, static_cast<char *>(workspace_p), &x);
    if ((a->n_q > 0 && !lse) || (need > 0 && (!workspace_p || ((uintptr_t)workspace_p & 15)))) return TL_EINVAL;
    if (need > workspace_bytes) return TL_ELIMIT;
    x.o = AttTensor{o->p, o->row, o->head};
    x.d_o = AttTensor{d_o->p, d_o->row, d_o->head};
    x.d_q = AttTensor{d_q->p, d_q->row, d_q->head};
    x.d_k = AttTensor{d_k->p, d_k->row, d_k->head};
    x.d_v = AttTensor{d_v->p, d_v->row, d_v->head};
    x.lse = const_cast<float *>(lse);
    x.vec = x.vec && in_pieces(*o, dt, D, 16) && in_pieces(*d_o, dt, D, 16);
    x.near = x.near && d_o->row < (1 << 20) && d_o->head < (1 << 20);
    x.vec_out = pieces_of_4(*d_q, dt, D) && pieces_of_4(*d_k, dt, D) && pieces_of_4(*d_v, dt, D);
    const hipStream_t st = (hipStream_t)hip_stream;
    const hipError_t e = dt == TL_DT_F32 ? attend_backward<float>(x, p, st) : dt == TL_DT_BF16 ? attend_backward<bf16_t>(x, p, st) : attend_backward<f16_t>(x, p, st);
    return e == hipSuccess ? TL_OK : TL_EHIP;
}

int tl_sample(int dtype, int n_rows, int vocab, const void *logits, int64_t row, const float *u, const float *temperature, const int32_t *top_k,
              const float *top_p, const float *min_p, int32_t *token, float *logprob, int32_t *kept, void *hip_stream)
{
    if (dtype < TL_DT_F32 || dtype > TL_DT_F16 || n_rows < 0 || vocab < 1 || vocab > (1 << 30)) return TL_EINVAL;
    if (n_rows == 0) return TL_OK;
    if (!logits || !u || !token || row < 0 || ((uintptr_t)logits & (element_size(dtype) - 1))) return TL_EINVAL;
    SampleArgs a = {};
    a.logits = logits;
    a.row = row;
    a.u = u;
    a.temperature = temperature;
    a.top_k = top_k;
    a.top_p = top_p;
    a.min_p = min_p;
    a.token = token;
    a.logprob = logprob;
    a.kept = kept;
    a.vocab = vocab;
    int bits = 0;
    while ((1ll << bits) < vocab) ++bits;
    a.shift = 62 - bits < 51 ? 62 - bits : 51;
    const hipStream_t st = (hipStream_t)hip_stream;
    const hipError_t e = dtype == TL_DT_F32 ? sample<float>(a, n_rows, st) : dtype == TL_DT_BF16 ? sample<bf16_t>(a, n_rows, st) : sample<f16_t>(a, n_rows, st);
    return e == hipSuccess ? TL_OK : TL_EHIP;
}

}  // extern "C"
