// Host side of the linear-attention entry points of include/gka.h: argument checks, launch plans, workspace carving.
// No device allocation, no synchronisation, nothing kept between calls.
#include "../../include/gka.h"
#include "gka_kernels.hpp"
#include "gka_linear.hpp"

namespace {

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// A walk is cut into segments up to this many workgroups of it: four for each CU, two of which run at a time.
constexpr int64_t kWalkWorkgroups = 4 * gka::kComputeUnits;

// Up to this many segments a walk adds up the states of those before it by itself; above, a launch between (the scan) does. The three
// walks of the backward pass, one of which reads the states transposed, add up 65536 floats at most, or 4 segments. Measured, us, added
// up against scanned (one chunk to a segment): forward pass, 8 states of 128 x 128, 16 segments 22.3 : 24.6; backward pass 62.8 : 47.1, 8
// segments 40.6 : 36.8, 16 such states, 16 segments 97 : 58; 16 states of 64 x 64, 16 segments 38.3 : 41.1; 8 of 256 x 128, 12 segments
// 98 : 62, 5 60 : 52.
constexpr int kMostSegmentsAddedUp = 16;
int most_added_up_backward(int64_t state_floats)
{
    const int64_t segs = 65536 / state_floats;
    return segs < 4 ? 4 : segs > kMostSegmentsAddedUp ? kMostSegmentsAddedUp : (int)segs;
}

// Threads of a launch, in each direction of its grid, have to be fewer.
constexpr int64_t kGridThreads = (int64_t)1 << 32;
// Tokens: positions up to two chunks behind the last one, and the end of its part of a sum over the sequence, are 32-bit numbers.
constexpr int kMaxTokens = 0x7fffe000;

struct Sizes {
    int share, G;
    int64_t pairs;
    bool bf16;
    gka::RowTensor q, k, v, o;    // strides only
};

enum class Call { kWalk, kDecode, kShared };

// Strides of one tensor [B, T, heads, d]; all zero: packed. The walks address a chunk's rows with 32-bit byte offsets; the calls for
// single tokens use 64 bits, and of one token the stride to the next is not used at all.
gka_status row_strides(const int64_t (&given)[3], const gka_linear_params *p, Call call, int T, int heads, int d, gka::RowTensor *x)
{
    constexpr int64_t kChunkRows = 1 << 23;
    const bool chunks = call == Call::kWalk && T > 1;
    x->p = nullptr;
    x->sh = d;
    x->st = (int64_t)heads * d;
    x->sb = (int64_t)T * heads * d;
    if (given[0] != 0 || given[1] != 0 || given[2] != 0) {
        const int piece = p->io_dtype == GKA_BF16 ? 8 : 4;        // rows are read and written 16 bytes at a time
        for (int64_t s : given)
            if (s <= 0 || s % piece) return GKA_ERR_SHAPE;
        if ((heads > 1 && given[2] < d) || (T > 1 && given[1] < d)) return GKA_ERR_SHAPE;
        x->sb = given[0];
        x->st = given[1];
        x->sh = given[2];
    }
    if (T == 1) x->st = d;
    return chunks && x->st >= kChunkRows ? GKA_ERR_UNSUPPORTED : GKA_OK;
}

gka_status check(const gka_linear_params *p, Call call, Sizes *s)
{
    if (!p) return GKA_ERR_NULL;
    if (p->B <= 0 || p->H <= 0 || p->H_kv <= 0 || p->H % p->H_kv) return GKA_ERR_SHAPE;
    if (call != Call::kShared && (p->T <= 0 || p->T > kMaxTokens)) return GKA_ERR_SHAPE;
    if (call == Call::kShared && (p->cache_tokens <= 0 || p->cache_tokens > kMaxTokens)) return GKA_ERR_SHAPE;
    if (p->d_k <= 0 || p->d_v <= 0) return GKA_ERR_SHAPE;
    if (p->d_k % 16 || p->d_v % 16 || p->d_k > 256 || p->d_v > 256) return GKA_ERR_UNSUPPORTED;
    if (p->io_dtype != GKA_F32 && p->io_dtype != GKA_BF16) return GKA_ERR_UNSUPPORTED;
    if (p->gate_per_head != 0 && p->gate_per_head != 1) return GKA_ERR_UNSUPPORTED;
    if (p->share < 0 || p->walk_chunks < 0) return GKA_ERR_SHAPE;
    if (p->reserved != 0) return GKA_ERR_UNSUPPORTED;
    s->share = p->share > 0 ? p->share : 1;
    if (p->B % s->share) return GKA_ERR_SHAPE;
    s->G = p->H / p->H_kv;
    s->pairs = (int64_t)p->B * p->H_kv;
    s->bf16 = p->io_dtype == GKA_BF16;
    // (of decode up to eight workgroups of 256 threads for a state where there are this many, of the shared call one of 512 for 16 heads)
    if (s->pairs >= (int64_t)1 << 21 || (int64_t)p->B * p->H > (int64_t)1 << 26) return GKA_ERR_SHAPE;
    const int T = call == Call::kShared ? 1 : p->T;
    gka_status e = row_strides(p->q_stride, p, call, T, p->H, p->d_k, &s->q);
    if (e == GKA_OK) e = row_strides(p->k_stride, p, call, T, p->H_kv, p->d_k, &s->k);
    if (e == GKA_OK) e = row_strides(p->v_stride, p, call, T, p->H_kv, p->d_v, &s->v);
    if (e == GKA_OK) e = row_strides(p->o_stride, p, call, T, p->H, p->d_v, &s->o);
    return e;
}

bool misaligned(std::initializer_list<const void *> pointers)
{
    for (const void *x : pointers)
        if ((uintptr_t)x & 15) return true;
    return false;
}

gka::RowTensor at(const void *p, gka::RowTensor strides)
{
    strides.p = p;
    return strides;
}

// ---- launch plan of a walk ----
struct WalkPlan {
    gka::LinearShape shape;
    int n_segs, seg_chunks;
    bool scanned;                      // the scan adds up the segments' states
    size_t state_bytes, decay_bytes;   // of the segments' states and decays in the workspace
};

// What a pass does over its chunks: `walks` walks in one launch, each chunk at walk_cost, after `summaries` in another, at summary_cost
// (in times of a chunk of the forward pass's summary, 1.7 us at d 128). The costs are those of bf16 tensors at d 128.
struct PassCost {
    int walks, summaries, most_added_up;
    float walk_cost, summary_cost;
};
PassCost forward_cost(int G) { return {1, 1, kMostSegmentsAddedUp, 1.9f + 0.85f * G, 1.0f}; }
PassCost backward_cost(int G, int64_t state_floats) { return {3, 2, most_added_up_backward(state_floats), 2.4f + 1.1f * G, 1.3f}; }

// Chunks of a segment, of `states` states of `chunks` chunks: the number whose estimated time is shortest. A chunk costs a CU the same
// whether one or two workgroups share it, so a launch takes ceil(workgroups / 256) segments' times, and the most segments for each
// such number are the candidates; the summaries walk all segments but the last once more; starting workgroups, the launches and adding
// up the states before a segment, or the scan, cost the rest. Measured, us, by chunks of a segment: 64 states
// x 4096 tokens, forward pass 4: 138, 8: 115, 16: 115, 32: 199, backward pass 8: 371, 16: 334, 32: 384; 8 states x 4 heads x 32768 tokens
// 8: 277, 16: 296, 32: 523; backward pass of 8 states x 3 heads x 1337 tokens 1: 71, 2: 82, 3: 110; float32, 16 states x 1001 tokens
// 1: 37, 2: 29, 4: 38.
int walk_segment(int64_t states, int64_t chunks, const PassCost &c)
{
    const auto rounds = [](int64_t workgroups) { return (float)((workgroups + gka::kComputeUnits - 1) / gka::kComputeUnits); };
    int64_t best = chunks;
    float best_time = -1.0f;
    const auto consider = [&](int64_t segs) {
        if (segs > chunks) segs = chunks;
        if (segs > 1 && segs * states > kWalkWorkgroups) return;
        const int64_t len = (chunks + segs - 1) / segs, n = (chunks + len - 1) / len;
        const float r = rounds(n * states * c.walks);
        float time = (r == 1.0f ? 1.08f : 1.0f) * r * len * c.walk_cost + 2.0f + r;   // (one workgroup on a CU: slower)
        if (n > 1)
            time += rounds((n - 1) * states * c.summaries) * len * c.summary_cost + 3.5f + (n > c.most_added_up ? 6.0f : 0.4f * n);
        if (best_time >= 0.0f && time >= best_time) return;
        best = len;
        best_time = time;
    };
    consider(1);
    consider(c.most_added_up);
    for (int r = 1; r <= c.walks * (int)(kWalkWorkgroups / gka::kComputeUnits); ++r) {
        const int64_t segs = r * gka::kComputeUnits / (states * c.walks);
        if (segs > 1) consider(segs);
    }
    return (int)best;
}

// like: a walk with the same segments (null: none).
gka_status plan_walk(const gka_linear_params *p, const Sizes &s, int dk, int dv, const PassCost &cost, const WalkPlan *like, WalkPlan *w)
{
    w->shape = gka::linear_shape(s.bf16, dk, dv);
    const int64_t chunks = ((int64_t)p->T + w->shape.chunk - 1) / w->shape.chunk;
    if (like) w->seg_chunks = like->seg_chunks;
    else if (p->walk_chunks > 0) w->seg_chunks = p->walk_chunks < chunks ? p->walk_chunks : (int)chunks;
    else w->seg_chunks = walk_segment(s.pairs * w->shape.slices, chunks, cost);
    w->n_segs = (int)((chunks + w->seg_chunks - 1) / w->seg_chunks);
    w->scanned = w->n_segs > cost.most_added_up;
    const int64_t states = s.pairs * w->shape.slices * w->n_segs;
    // (three walks of 512 threads are one launch; the scan: a thread for four floats of a state)
    if (states * 3 * 512 >= kGridThreads) return GKA_ERR_SHAPE;
    if (w->n_segs > 1 && s.pairs * w->shape.slices * (w->shape.state_floats / 4) >= kGridThreads) return GKA_ERR_SHAPE;
    w->state_bytes = w->n_segs > 1 ? align_up((size_t)states * w->shape.state_floats * sizeof(float), 256) : 0;
    w->decay_bytes = w->n_segs > 1 ? align_up((size_t)s.pairs * w->n_segs * sizeof(float), 256) : 0;
    return GKA_OK;
}

gka::LinearWalkArgs walk_args(const gka_linear_params *p, const Sizes &s, const WalkPlan &w, const float *gate, int dk, int dv, char *ws)
{
    gka::LinearWalkArgs a = {};
    a.gate = gate;
    a.gate_per_head = p->gate_per_head;
    a.B = p->B; a.T = p->T; a.Hkv = p->H_kv;
    a.n_q = a.n_src = 1;
    a.dk = dk; a.dv = dv;
    a.share = 1;
    a.n_segs = w.n_segs; a.seg_chunks = w.seg_chunks;
    a.scanned = w.scanned;
    a.slices = w.shape.slices;
    a.seg_states = (float *)ws;
    a.seg_decay = (float *)(ws + w.state_bytes);
    return a;
}

struct BackwardPlan {
    Sizes s;
    WalkPlan q, k, v;                  // the walks of dq, dk, dv
    size_t off_q, off_k, off_q_dot, off_k_dot, off_state_dot, off_gate, off_states, off_S_chunk, off_dS_chunk, off_small, total;
};

gka_status plan_backward(const gka_linear_params *p, BackwardPlan *b)
{
    gka_status e = check(p, Call::kWalk, &b->s);
    if (e != GKA_OK) return e;
    // (the walks of dk and dv have their segments in common)
    const PassCost cost = backward_cost(b->s.G, gka::linear_shape(b->s.bf16, p->d_v, p->d_k).state_floats);
    if ((e = plan_walk(p, b->s, p->d_v, p->d_k, cost, nullptr, &b->q)) != GKA_OK) return e;
    b->k = b->q;
    if ((e = plan_walk(p, b->s, p->d_k, p->d_v, cost, &b->q, &b->v)) != GKA_OK) return e;
    size_t off = 0;
    b->off_q = off; off += b->q.state_bytes + b->q.decay_bytes;
    b->off_k = off; off += b->k.state_bytes + b->k.decay_bytes;
    // (a thread for four tokens of a state, in parts of 4096; a thread for four floats of the states)
    if (b->s.pairs * ((p->T + (int64_t)4095) / 4096) * 1024 >= kGridThreads || b->s.pairs * p->d_k * p->d_v / 4 >= kGridThreads)
        return GKA_ERR_SHAPE;
    const size_t tokens = (size_t)b->s.pairs * p->T;
    b->off_q_dot = off; off += align_up(b->q.shape.slices * tokens * b->s.G * sizeof(double), 256);
    b->off_k_dot = off; off += align_up(b->k.shape.slices * tokens * sizeof(double), 256);
    b->off_state_dot = off; off += align_up(b->q.shape.slices * b->s.pairs * sizeof(double), 256);
    b->off_gate = off; off += align_up(gka::linear_gate_workspace_bytes(b->s.pairs, p->T, b->q.shape.chunk), 256);
    // (two states for each chunk: which ones hold small gates, the host does not know)
    const size_t chunks = (size_t)b->s.pairs * (((int64_t)p->T + b->q.shape.chunk - 1) / b->q.shape.chunk);
    b->off_S_chunk = off; off += chunks * b->q.shape.slices * b->q.shape.state_floats * sizeof(float);
    b->off_dS_chunk = off; off += chunks * b->q.shape.slices * b->q.shape.state_floats * sizeof(float);
    b->off_small = off; off += align_up(chunks * sizeof(int), 256);
    b->off_states = off;
    // (room for a state of every sequence whether or not initial states are shared: one size for all calls)
    off += align_up((size_t)b->s.pairs * p->d_k * p->d_v * sizeof(float), 256);
    b->total = off;
    return GKA_OK;
}

}  // namespace

namespace gka {

LinearShape linear_shape(bool bf16, int dk, int dv)
{
    LinearShape s;
    s.chunk = bf16 ? 64 : 32;
    s.slice = dv <= 64 ? 64 : 128;
    s.padded_dk = dk <= 64 ? 64 : dk <= 128 ? 128 : 256;
    s.slices = (dv + s.slice - 1) / s.slice;
    s.state_floats = (int64_t)s.slice * s.padded_dk;
    return s;
}

hipError_t launch_linear_forward(const LinearWalkArgs &a, bool bf16, hipStream_t stream)
{
    switch (linear_shape(bf16, a.dk, a.dv).padded_dk) {
    case 64: return bf16 ? launch_linear_forward_bf16_64(a, stream) : launch_linear_forward_f32_64(a, stream);
    case 128: return bf16 ? launch_linear_forward_bf16_128(a, stream) : launch_linear_forward_f32_128(a, stream);
    default: return bf16 ? launch_linear_forward_bf16_256(a, stream) : launch_linear_forward_f32_256(a, stream);
    }
}

hipError_t launch_linear_backward(const LinearWalkArgs &dq, const LinearWalkArgs &dk, const LinearWalkArgs &dv, bool bf16, hipStream_t stream)
{
    const LinearShape of_dk = linear_shape(bf16, dk.dk, dk.dv), of_dv = linear_shape(bf16, dv.dk, dv.dv);
    LinearWalkArgs v = dv;
    v.seg_states = dk.seg_states;
    v.seg_decay = dk.seg_decay;
    v.seg_turned[0] = of_dk.slice / 16;
    v.seg_turned[1] = of_dk.padded_dk / 16;
    v.seg_turned[2] = of_dk.slices;
    const bool alike = of_dk.padded_dk == of_dv.padded_dk && of_dk.slice == of_dv.slice && of_dk.slices == of_dv.slices;
    hipError_t e;
    switch (of_dk.padded_dk) {
    case 64: e = bf16 ? launch_linear_backward_bf16_64(dq, dk, v, alike, stream) : launch_linear_backward_f32_64(dq, dk, v, alike, stream); break;
    case 128: e = bf16 ? launch_linear_backward_bf16_128(dq, dk, v, alike, stream) : launch_linear_backward_f32_128(dq, dk, v, alike, stream); break;
    default: e = bf16 ? launch_linear_backward_bf16_256(dq, dk, v, alike, stream) : launch_linear_backward_f32_256(dq, dk, v, alike, stream);
    }
    if (e != hipSuccess || alike) return e;
    switch (of_dv.padded_dk) {
    case 64: return bf16 ? launch_linear_values_bf16_64(v, stream) : launch_linear_values_f32_64(v, stream);
    case 128: return bf16 ? launch_linear_values_bf16_128(v, stream) : launch_linear_values_f32_128(v, stream);
    default: return bf16 ? launch_linear_values_bf16_256(v, stream) : launch_linear_values_f32_256(v, stream);
    }
}

}  // namespace gka

extern "C" {

size_t gka_linear_forward_workspace_bytes(const gka_linear_params *p)
{
    Sizes s;
    WalkPlan w;
    if (check(p, Call::kWalk, &s) != GKA_OK || plan_walk(p, s, p->d_k, p->d_v, forward_cost(s.G), nullptr, &w) != GKA_OK) return 0;
    const size_t bytes = w.state_bytes + w.decay_bytes;
    return bytes > 0 ? bytes : 256;
}

gka_status gka_linear_forward(const gka_linear_params *p, const void *q, const void *k, const void *v, const float *gate, void *o,
                              const float *S_init, float *S_final, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    Sizes s;
    WalkPlan w;
    gka_status e = check(p, Call::kWalk, &s);
    if (e != GKA_OK) return e;
    if ((e = plan_walk(p, s, p->d_k, p->d_v, forward_cost(s.G), nullptr, &w)) != GKA_OK) return e;
    if (!q || !k || !v || !gate || !o) return GKA_ERR_NULL;
    if (misaligned({q, k, v, o, S_init, S_final})) return GKA_ERR_SHAPE;
    if (S_final && S_final == S_init && s.share > 1) return GKA_ERR_SHAPE;   // (states that other sequences still read)
    const size_t need = w.state_bytes + w.decay_bytes;
    if (need > 0 && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255))) return GKA_ERR_WORKSPACE;
    gka::LinearWalkArgs a = walk_args(p, s, w, gate, p->d_k, p->d_v, (char *)workspace);
    a.q = at(q, s.q); a.k = at(k, s.k); a.v = at(v, s.v); a.y = at(o, s.o);
    a.n_q = s.G;
    a.init = S_init; a.share = s.share;
    a.final = S_final;
    // (the last segment of a sequence may write its state before another one has started: in place only the scan reads the old states)
    if (S_final && S_final == S_init && a.n_segs > 1) a.scanned = 1;
    return gka::launch_linear_forward(a, s.bf16, (hipStream_t)hip_stream) == hipSuccess ? GKA_OK : GKA_ERR_LAUNCH;
}

size_t gka_linear_backward_workspace_bytes(const gka_linear_params *p)
{
    BackwardPlan b;
    return plan_backward(p, &b) == GKA_OK ? b.total : 0;
}

gka_status gka_linear_backward(const gka_linear_params *p, const void *q, const void *k, const void *v, const float *gate,
                               const void *dy, const float *S_init, const float *dS_final, void *dq, void *dk, void *dv, float *dgate,
                               float *dS_init, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    BackwardPlan b;
    gka_status e = plan_backward(p, &b);
    if (e != GKA_OK) return e;
    if (!q || !k || !v || !gate || !dy || !dq || !dk || !dv || !dgate) return GKA_ERR_NULL;
    if (misaligned({q, k, v, dy, S_init, dS_final, dq, dk, dv, dS_init})) return GKA_ERR_SHAPE;
    if (dS_init && (dS_init == S_init || dS_init == dS_final)) return GKA_ERR_SHAPE;   // (walks read those while another writes)
    if (!workspace || workspace_bytes < b.total || ((uintptr_t)workspace & 255)) return GKA_ERR_WORKSPACE;
    hipStream_t stream = (hipStream_t)hip_stream;
    char *ws = (char *)workspace;
    const Sizes &s = b.s;
    double *q_dot = (double *)(ws + b.off_q_dot), *k_dot = (double *)(ws + b.off_k_dot), *state_dot = (double *)(ws + b.off_state_dot);
    const int64_t none[3] = {0, 0, 0};
    gka::RowTensor packed_q, packed_k, packed_v;
    (void)row_strides(none, p, Call::kWalk, p->T, p->H, p->d_k, &packed_q);
    (void)row_strides(none, p, Call::kWalk, p->T, p->H_kv, p->d_k, &packed_k);
    (void)row_strides(none, p, Call::kWalk, p->T, p->H_kv, p->d_v, &packed_v);
    // dq_t = S_t^T dy_t
    gka::LinearWalkArgs wq = walk_args(p, s, b.q, gate, p->d_v, p->d_k, ws + b.off_q);
    wq.q = at(dy, s.o); wq.k = at(v, s.v); wq.v = at(k, s.k); wq.y = at(dq, packed_q);
    wq.n_q = s.G;
    wq.init = S_init; wq.share = s.share; wq.transposed = 1;
    wq.dot_with = at(q, s.q); wq.dot_out = q_dot;
    wq.chunk_states = (float *)(ws + b.off_S_chunk); wq.small_gates = (int *)(ws + b.off_small);
    if (dS_final) {
        wq.state_dot_with = dS_final;
        wq.state_dot_out = state_dot;
    }
    // dk_t = dS_t^T v_t, dS_t = sum_g dy_t q_t^T + gate_{t+1} dS_{t+1}
    gka::LinearWalkArgs wk = walk_args(p, s, b.k, gate, p->d_v, p->d_k, ws + b.off_k);
    wk.q = at(v, s.v); wk.k = at(dy, s.o); wk.v = at(q, s.q); wk.y = at(dk, packed_k);
    wk.n_src = s.G;
    wk.reverse = 1;
    wk.init = dS_final; wk.transposed = 1;
    wk.dot_with = at(k, s.k); wk.dot_out = k_dot;
    wk.chunk_states = (float *)(ws + b.off_dS_chunk);
    // dv_t = dS_t k_t
    gka::LinearWalkArgs wv = walk_args(p, s, b.v, gate, p->d_k, p->d_v, ws + b.off_k);
    wv.q = at(k, s.k); wv.k = at(q, s.q); wv.v = at(dy, s.o); wv.y = at(dv, packed_v);
    wv.n_src = s.G;
    wv.reverse = 1;
    wv.init = dS_final;
    wv.final = dS_init && s.share > 1 ? (float *)(ws + b.off_states) : dS_init;
    wv.final_times_gate = 1;
    if (gka::launch_linear_backward(wq, wk, wv, s.bf16, stream) != hipSuccess) return GKA_ERR_LAUNCH;
    if (dS_init && s.share > 1 &&
        gka::launch_linear_state_sum(wv.final, dS_init, p->B / s.share, s.share, (int64_t)p->H_kv * p->d_k * p->d_v, stream) != hipSuccess)
        return GKA_ERR_LAUNCH;
    gka::LinearGateArgs g = {};
    g.q_dq = q_dot; g.k_dk = k_dot; g.state_dot = dS_final ? state_dot : nullptr;
    g.q_slices = b.q.shape.slices; g.k_slices = b.k.shape.slices; g.G = s.G;
    g.gate = gate; g.dgate = dgate; g.gate_per_head = p->gate_per_head;
    g.B = p->B; g.T = p->T; g.Hkv = p->H_kv;
    g.q = wq.dot_with; g.k = wk.dot_with; g.v = wk.q; g.dy = wq.q;
    g.dk = p->d_k; g.dv = p->d_v; g.chunk = b.q.shape.chunk;
    g.small_gates = wq.small_gates; g.S_chunk = wq.chunk_states; g.dS_chunk = wk.chunk_states;
    g.state_slice = b.q.shape.slice; g.state_dk = b.q.shape.padded_dk;
    return gka::launch_linear_gate(g, s.bf16, ws + b.off_gate, stream) == hipSuccess ? GKA_OK : GKA_ERR_LAUNCH;
}

gka_status gka_linear_decode(const gka_linear_params *p, const float *S_in, float *S_out, const void *q, const void *k, const void *v,
                             const float *gate, void *o, void *hip_stream)
{
    Sizes s;
    gka_status e = check(p, Call::kDecode, &s);
    if (e != GKA_OK) return e;
    if (!S_in || !S_out || !q || !k || !v || !gate || !o) return GKA_ERR_NULL;
    if (misaligned({S_in, S_out, q, k, v, o})) return GKA_ERR_SHAPE;
    if (S_in == S_out && s.share > 1) return GKA_ERR_SHAPE;
    gka::LinearDecodeArgs a = {};
    a.S_in = S_in; a.S_out = S_out;
    a.q = at(q, s.q); a.k = at(k, s.k); a.v = at(v, s.v); a.y = at(o, s.o);
    a.gate = gate; a.gate_per_head = p->gate_per_head;
    a.share = s.share; a.B = p->B; a.T = p->T; a.Hkv = p->H_kv; a.G = s.G; a.dk = p->d_k; a.dv = p->d_v;
    return gka::launch_linear_decode(a, s.bf16, (hipStream_t)hip_stream) == hipSuccess ? GKA_OK : GKA_ERR_LAUNCH;
}

gka_status gka_linear_decode_shared(const gka_linear_params *p, const float *S_prefix, const void *q, const void *k, const void *v,
                                    const float *gate, void *k_cache, void *v_cache, float *gate_cache, const int32_t *lengths, void *o,
                                    void *hip_stream)
{
    Sizes s;
    gka_status e = check(p, Call::kShared, &s);
    if (e != GKA_OK) return e;
    if (!S_prefix || !q || !k || !v || !gate || !k_cache || !v_cache || !lengths || !o) return GKA_ERR_NULL;
    if (!gate_cache && !p->gate_per_head) return GKA_ERR_NULL;
    if (misaligned({S_prefix, q, k, v, k_cache, v_cache, o})) return GKA_ERR_SHAPE;
    gka::LinearSharedArgs a = {};
    a.S = S_prefix;
    a.q = at(q, s.q); a.k = at(k, s.k); a.v = at(v, s.v); a.y = at(o, s.o);
    a.gate = gate; a.gate_per_head = p->gate_per_head;
    a.k_cache = k_cache; a.v_cache = v_cache; a.gate_cache = p->gate_per_head ? nullptr : gate_cache; a.lengths = lengths;
    a.share = s.share; a.B = p->B; a.N = p->cache_tokens; a.Hkv = p->H_kv; a.G = s.G; a.dk = p->d_k; a.dv = p->d_v;
    return gka::launch_linear_shared(a, s.bf16, (hipStream_t)hip_stream) == hipSuccess ? GKA_OK : GKA_ERR_LAUNCH;
}

}  // extern "C"
