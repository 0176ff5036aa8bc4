// C entry points of the recurrence along sentences.
#include "entry.hpp"
#include "recur.hpp"

using namespace tl;

namespace {

constexpr int WAVES = 8, ROWS = 8;              // of a block: 64 words
// (as many words as a state's place and the block behind the last word can be counted in 32 bits with)
constexpr int MOST_ROWS = INT32_MAX - 65536;

// Channels of a lane: 8 bytes of a row forwards, 4 or 8 backwards (four tensors' worth of registers).
constexpr int lanes_channels(int size, bool back) { return back ? 2 : 8 / size; }

bool check(const tl_recurrence *r)
{
    if (!r || !is_dtype(r->dtype) || (r->gate != TL_GATE_SIGMOID && r->gate != TL_GATE_GIVEN)) return false;
    if (r->n_trees < 0 || r->n_rows < 0 || r->n_rows > MOST_ROWS || r->channels < 1 || r->channels > (1 << 20)) return false;
    if (r->n_trees == 0) return r->n_rows == 0;
    return r->off && check_matrix(r->g, r->g_row, r->dtype, r->n_rows, r->channels, false) && check_matrix(r->x, r->x_row, r->dtype, r->n_rows, r->channels, false);
}

struct Plan {
    int V, slices, shift, slots;
    bool single;                                // a wave per sentence
    long long blocks;
};

bool plan(const tl_recurrence *r, bool back, Plan *p)
{
    p->V = lanes_channels(element_size(r->dtype), back);
    if (r->channels < p->V) p->V = 1;
    p->slices = (r->channels + 64 * p->V - 1) / (64 * p->V);
    const long long rows = r->n_rows, trees = r->n_trees;
    p->single = !back && rows <= 8 * trees;
    p->shift = REC_WHOLE;
    const long long wanted = 2ll * compute_units();
    if (trees * p->slices < wanted && rows > 128 * trees) {
        p->shift = 6;
        while (p->shift < 14 && (rows >> (p->shift + 1)) * p->slices >= 2 * wanted) ++p->shift;
    }
    const long long slots = (rows >> p->shift) + trees;
    p->blocks = slots * p->slices;
    p->slots = (int)slots;
    return p->blocks <= most_blocks(64 * WAVES);
}

long long workspace(const tl_recurrence *r, const Plan &p) { return p.shift == REC_WHOLE ? 0 : round16(8ll * p.slots * r->channels); }

RecurArgs arguments(const tl_recurrence *r, const Plan &p)
{
    RecurArgs a = {};
    a.g = r->g;
    a.g_row = r->g_row;
    a.x = r->x;
    a.x_row = r->x_row;
    a.off = r->off;
    a.n_trees = r->n_trees;
    a.n_rows = r->n_rows;
    a.C = r->channels;
    a.slices = p.slices;
    a.slots = p.slots;
    a.shift = p.shift;
    return a;
}

template <typename T, int V, int GATE> hipError_t forward_of(const RecurArgs &a, const Plan &p, hipStream_t st)
{
    if (p.shift != REC_WHOLE) {
        hipLaunchKernelGGL((k_recur_pairs<T, V, WAVES, ROWS, GATE, false>), dim3((unsigned)p.blocks), dim3(64 * WAVES), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (p.single) hipLaunchKernelGGL((k_recur<T, V, 1, ROWS, GATE>), dim3((unsigned)p.blocks), dim3(64), 0, st, a);
    else hipLaunchKernelGGL((k_recur<T, V, WAVES, ROWS, GATE>), dim3((unsigned)p.blocks), dim3(64 * WAVES), 0, st, a);
    return hipGetLastError();
}

template <typename T, int V, int GATE> hipError_t backward_of(const RecurArgs &a, const Plan &p, hipStream_t st)
{
    if (p.shift != REC_WHOLE) {
        hipLaunchKernelGGL((k_recur_pairs<T, V, WAVES, ROWS, GATE, true>), dim3((unsigned)p.blocks), dim3(64 * WAVES), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((k_recur_back<T, V, WAVES, ROWS, GATE>), dim3((unsigned)p.blocks), dim3(64 * WAVES), 0, st, a);
    return hipGetLastError();
}

template <typename T, int GATE> hipError_t launch_at(const RecurArgs &a, const Plan &p, bool back, hipStream_t st)
{
    constexpr int F = lanes_channels(sizeof(T), false), B = lanes_channels(sizeof(T), true);
    if (back) return p.V == 1 ? backward_of<T, 1, GATE>(a, p, st) : backward_of<T, B, GATE>(a, p, st);
    return p.V == 1 ? forward_of<T, 1, GATE>(a, p, st) : forward_of<T, F, GATE>(a, p, st);
}

template <typename T> hipError_t launch_for(const RecurArgs &a, int gate, const Plan &p, bool back, hipStream_t st)
{
    return gate == TL_GATE_SIGMOID ? launch_at<T, TL_GATE_SIGMOID>(a, p, back, st) : launch_at<T, TL_GATE_GIVEN>(a, p, back, st);
}

int launch(const tl_recurrence *r, const RecurArgs &a, const Plan &p, bool back, void *stream)
{
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = r->dtype == TL_DT_F32    ? launch_for<float>(a, r->gate, p, back, st)
                         : r->dtype == TL_DT_BF16 ? launch_for<bf16_t>(a, r->gate, p, back, st)
                                                  : launch_for<f16_t>(a, r->gate, p, back, st);
    return e == hipSuccess ? TL_OK : TL_EHIP;
}

bool float_pointer(const void *p) { return ((uintptr_t)p & 3) == 0; }

}  // namespace

extern "C" {

int tl_recur_workspace(const tl_recurrence *r, int backward, int64_t *bytes)
{
    Plan p;
    if (!bytes || !check(r)) return TL_EINVAL;
    *bytes = 0;
    if (r->n_trees == 0) return TL_OK;
    if (!plan(r, backward != 0, &p)) return TL_EINVAL;
    *bytes = workspace(r, p);
    return TL_OK;
}

int tl_recur(const tl_recurrence *r, const float *h0, void *h, int64_t h_row, float *h_last, float *tape, void *workspace_p, int64_t workspace_bytes, void *hip_stream)
{
    if (!check(r) || !check_matrix(h, h_row, r->dtype, r->n_rows, r->channels, true)) return TL_EINVAL;
    if (!float_pointer(h0) || !float_pointer(h_last) || !float_pointer(tape)) return TL_EINVAL;
    if (r->n_trees == 0) return TL_OK;
    Plan p;
    if (!plan(r, false, &p)) return TL_EINVAL;
    const long long need = workspace(r, p);
    if (need > workspace_bytes) return TL_ELIMIT;
    if (need > 0 && (!workspace_p || ((uintptr_t)workspace_p & 15))) return TL_EINVAL;
    RecurArgs a = arguments(r, p);
    a.h = h;
    a.h_row = h_row;
    a.h0 = h0;
    a.h_last = h_last;
    a.tape = tape;
    a.pairs = static_cast<float *>(workspace_p);
    return launch(r, a, p, false, hip_stream);
}

int tl_recur_backward(const tl_recurrence *r, const float *tape, const void *d_h, int64_t d_h_row, const float *d_last, void *d_g, int64_t d_g_row, void *d_x,
                      int64_t d_x_row, float *d_h0, void *workspace_p, int64_t workspace_bytes, void *hip_stream)
{
    if (!check(r) || (d_h && !check_matrix(d_h, d_h_row, r->dtype, r->n_rows, r->channels, false))) return TL_EINVAL;
    if (!check_matrix(d_g, d_g_row, r->dtype, r->n_rows, r->channels, true) || !check_matrix(d_x, d_x_row, r->dtype, r->n_rows, r->channels, true)) return TL_EINVAL;
    if (!float_pointer(tape) || !float_pointer(d_last) || !float_pointer(d_h0) || (r->n_rows > 0 && !tape)) return TL_EINVAL;
    if (r->n_trees == 0) return TL_OK;
    Plan p;
    if (!plan(r, true, &p)) return TL_EINVAL;
    const long long need = workspace(r, p);
    if (need > workspace_bytes) return TL_ELIMIT;
    if (need > 0 && (!workspace_p || ((uintptr_t)workspace_p & 15))) return TL_EINVAL;
    RecurArgs a = arguments(r, p);
    a.tape = const_cast<float *>(tape);
    a.d_h = d_h;
    a.d_h_row = d_h_row;
    a.d_last = d_last;
    a.d_g = d_g;
    a.d_g_row = d_g_row;
    a.d_x = d_x;
    a.d_x_row = d_x_row;
    a.d_h0 = d_h0;
    a.pairs = static_cast<float *>(workspace_p);
    return launch(r, a, p, true, hip_stream);
}

}  // extern "C"
