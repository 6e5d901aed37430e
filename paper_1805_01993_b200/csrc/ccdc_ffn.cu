// Gated feed-forward block, forward and backward: what is computed in which order, where it is kept, and the small
// kernels around the products (copies into the layout the tensor cores read, sums of products cut along k).
#include <algorithm>

#include "ccdc_ffn.h"
#include "ccdc_ffn_mma.h"
#include "ccdc_ffn_rows.h"

namespace {

constexpr int MAX_COPIES = 5, MAX_JOINS = 4;

// ------------------------------------------------------------------ copies
// A matrix the tensor cores cannot read as it lies: rows that TMA cannot address (16-byte rule) are copied to padded
// rows; binary32 is split into three bf16 planes (see next_plane).  Bound by its bytes: the 13.6 M words of a binary32 block of
// 1024 x 4096 with 1024 rows in 33 us, 4.1 TB/s read and written.
struct Copy {
    const void *from;
    void *to;
    long long rows, cols, ld, ld_to;
};
struct Copies {
    Copy c[MAX_COPIES];
    int count, f32;
};
__global__ void __launch_bounds__(256) k_ffn_copy(const Copies a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const Copy &c = a.c[blockIdx.y];
    const long long pairs = c.ld_to / 2, n = c.rows * pairs;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < n; i += gridDim.x * 256LL) {
        const long long r = i / pairs, k = (i - r * pairs) * 2;
        if (k >= c.cols) continue;
        const bool two = k + 1 < c.cols;
        if (a.f32) {
            const float *p = static_cast<const float *>(c.from) + r * c.ld + k;
            float x = p[0], y = two ? p[1] : 0.0f;
            uint32_t *q = static_cast<uint32_t *>(c.to) + i;
            q[0] = fmaxf(fabsf(x), fabsf(y)) < FIRST_MOST && x == x && y == y ? next_plane(x, y) : first_plane_of_any(x, y);
            q[n] = next_plane(x, y), q[2 * n] = next_plane(x, y);
        } else {
            const uint16_t *p = static_cast<const uint16_t *>(c.from) + r * c.ld + k;
            static_cast<uint32_t *>(c.to)[i] = p[0] | (two ? (uint32_t)p[1] << 16 : 0u);
        }
    }
}

// ------------------------------------------------------------------ joins
// The sum of a product's parts along k, in order, four columns a thread.  The parts of a small product are still in L2:
// 512 x 1024 outputs take 3 to 5 us, most of it the launch.
struct Join {
    const float *parts;
    void *to;
    long long rows, cols, ld_parts, ld_to;
    int splits, type;
};
struct Joins {
    Join j[MAX_JOINS];
    int count;
};
__global__ void __launch_bounds__(256) k_ffn_join(const Joins a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const Join &j = a.j[blockIdx.y];
    const long long quads = (j.cols + 3) / 4, n = j.rows * quads, plane = j.rows * j.ld_parts;
    const bool wide = j.ld_to % 4 == 0 && (reinterpret_cast<uintptr_t>(j.to) & 15) == 0;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < n; i += gridDim.x * 256LL) {
        const long long r = i / quads, k = (i - r * quads) * 4;
        const float *p = j.parts + r * j.ld_parts + k;
        float4 v = *reinterpret_cast<const float4 *>(p);
        for (int s = 1; s < j.splits; ++s) {
            const float4 o = *reinterpret_cast<const float4 *>(p + s * plane);
            v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
        }
        const long long at = r * j.ld_to + k;
        if (wide && k + 4 <= j.cols) {
            if (j.type == CCDC_F32)
                *reinterpret_cast<float4 *>(static_cast<float *>(j.to) + at) = v;
            else
                *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(j.to) + at) =
                    j.type == CCDC_BF16 ? make_uint2(pack2<bf16>(v.x, v.y), pack2<bf16>(v.z, v.w))
                                        : make_uint2(pack2<fp16>(v.x, v.y), pack2<fp16>(v.z, v.w));
        } else {
            const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (k + e < j.cols) {
                    if (j.type == CCDC_F32)
                        static_cast<float *>(j.to)[at + e] = f[e];
                    else if (j.type == CCDC_BF16)
                        static_cast<bf16 *>(j.to)[at + e] = from_f32<bf16>(f[e]);
                    else
                        static_cast<fp16 *>(j.to)[at + e] = from_f32<fp16>(f[e]);
                }
        }
    }
}

template <class P>
int launch_small(void (*kernel)(P), const P &p, long long items, int rows, int sms, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)std::max<long long>(1, std::min<long long>((items + 255) / 256, 16LL * sms)), (unsigned)rows);
    cfg.blockDim = dim3(256);
    cfg.stream = s;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p);
    if (e != cudaSuccess) return ccdc_internal_cuda_fail((int)e);
    ccdc_internal_count_launch();
    return CCDC_OK;
}

// ------------------------------------------------------------------ layouts
long long pitch(long long cols) { return (long long)round_up((size_t)cols, 8); }
int planes_of(int dtype) { return dtype == CCDC_F32 ? 3 : 1; }
size_t inner_bytes(long long M, long long F, int dtype) {       // a, dh, du
    return round_up((size_t)planes_of(dtype) * M * pitch(F) * 2, 256);
}
size_t wide_bytes(long long M, long long F) {                   // h, u
    return round_up((size_t)((M + 31) / 32) * ffn_saved_groups(F) * 128 * sizeof(float), 256);
}
size_t copy_bytes(long long rows, long long cols, int dtype) {
    return round_up((size_t)planes_of(dtype) * rows * pitch(cols) * 2, 256);
}
bool readable(const void *p, long long ld, long long rows, int dtype) {
    return is_16bit(dtype) && aligned_to(p, 16) && (rows < 2 || ld % 8 == 0);
}

// the workspace, handed out front to back; a null base only counts
struct Space {
    char *base;
    size_t size = 0, used = 0;
    void *take(size_t bytes) {
        void *p = base ? base + used : nullptr;
        used += round_up(bytes, 256);
        return p;
    }
};

// ------------------------------------------------------------------ tiles and cuts
// How a launch's products are tiled, and how often each is cut along k.  The estimate, in cycles: a step of 64 k is
// bounded by the fetch of its blocks (48 KiB for the 256 x 512 tile, 72 KiB for binary32, 32 KiB for the others, at about
// 39 bytes a cycle); an item costs 2500 to begin, and its epilogue goes by 32-column pieces (two warps side by side),
// hidden under the next item's products unless the tile fills tensor memory; a cut product is written and read again in
// binary32 and needs another launch.
struct Shape {
    long long M, N, steps;      // steps of 64 k over all terms
    int splits;
};
MmaTile choose_tiles(Shape *q, int count, MmaEpilogue e, bool planes, int sms) {
    double best = 1e30;
    MmaTile tile = MMA_SINGLE;
    int cuts[4] = {};
    for (int shape = planes ? MMA_PLANES : MMA_WIDE; shape <= (planes ? MMA_PLANES : MMA_SINGLE); ++shape) {
        const MmaTile at = (MmaTile)shape;
        const long long rows = mma_tile_rows(at), cols = mma_tile_columns(at) / (e == MMA_GATE ? 2 : 1);
        const double step = planes ? 1890 : at == MMA_WIDE ? 1260 : 840, units = at == MMA_SINGLE ? sms : sms / 2;
        const double epilogue = cols / 64 * (e == MMA_STORE ? 400.0 : e == MMA_GATE ? 3000.0 : 3500.0);
        for (long long most = e == MMA_STORE ? 8 : 1LL << 40;; most = most >= 256 ? 1LL << 40 : most * 2) {
            double total = 0, longest = 0, items = 0, parts = 0;
            int c[4];
            for (int i = 0; i < count; ++i) {
                const long long tiles = ((q[i].M + rows - 1) / rows) * ((q[i].N + cols - 1) / cols);
                c[i] = (int)std::min<long long>(std::max<long long>(1, (q[i].steps + most / 2) / most), 64);
                const double work = (double)q[i].steps / c[i] * step + 500;
                const double cost = at == MMA_WIDE ? work + epilogue : std::max(work, epilogue);
                total += cost * tiles * c[i], items += (double)tiles * c[i];
                longest = std::max(longest, cost);
                if (c[i] > 1) parts += 8.0 * c[i] * q[i].M * q[i].N;
            }
            double t = items <= units ? longest : std::max(longest, total / units) + longest / 2;
            t += 2500 + (at == MMA_WIDE ? 0 : epilogue);
            if (parts > 0) t += 5000 + parts / 2000;        // parts mostly stay in L2
            if (t < best) {
                best = t, tile = at;
                for (int i = 0; i < count; ++i) cuts[i] = c[i];
            }
            if (most >= 1LL << 40) break;
        }
    }
    for (int i = 0; i < count; ++i) q[i].splits = cuts[i];
    return tile;
}

long long steps_of(long long K, int terms) { return (K + 63) / 64 * terms; }

int check_ffn(long long M, long long D, long long F, int dtype, int act) {
    if (M < 0 || D < 1 || F < 1 || !is_float_type(dtype) || act < CCDC_ACT_SILU || act > CCDC_ACT_RELU) return CCDC_EINVAL;
    if (M > (1LL << 21) || D > (1LL << 20) || F > (1LL << 20)) return CCDC_ESIZE;
    return CCDC_OK;
}

// One call: the operands as the tensor cores read them, the workspace, the launches.  With plan_only set the same
// steps only count the workspace and run nothing.
struct Call {
    long long M, D, F;
    int dtype, act, sms;
    bool plan_only, aligned;
    Space space;
    cudaStream_t s;
    Copies copies = {};
    Joins joins = {};
    int rc = CCDC_OK;

    int type() const { return dtype == CCDC_F16 ? CCDC_F16 : CCDC_BF16; }

    MmaMatrix operand(const void *p, long long rows, long long cols, long long ld) {
        const bool direct = plan_only ? aligned && is_16bit(dtype) : readable(p, ld, rows, dtype);
        if (direct) return {p, rows, cols, rows < 2 ? pitch(cols) : ld, 1};
        void *to = space.take(copy_bytes(rows, cols, dtype));
        copies.c[copies.count++] = {p, to, rows, cols, ld, pitch(cols)};
        return {to, rows, cols, pitch(cols), planes_of(dtype)};
    }
    // everything is laid out: does it fit?
    bool fits() {
        if (plan_only) return false;
        if (space.used > space.size) rc = CCDC_ESIZE;
        return rc == CCDC_OK;
    }
    void run_copies() {
        if (!copies.count || rc != CCDC_OK) return;
        copies.f32 = dtype == CCDC_F32;
        long long most = 0;
        for (int i = 0; i < copies.count; ++i) most = std::max(most, copies.c[i].rows * copies.c[i].ld_to / 2);
        rc = launch_small(k_ffn_copy, copies, most, copies.count, sms, s);
    }
    MmaMatrix inner(void *p) const { return {p, M, F, pitch(F), planes_of(dtype)}; }
    // where a product goes: its output, or parts of it to be joined
    void to_output(MmaProduct &q, int splits, void *c, long long ldc, int c_type) {
        q.splits = splits;
        q.c = c, q.ldc = ldc, q.c_type = c_type;
        if (splits == 1) return;
        q.ldc = (q.N + 3) / 4 * 4;
        q.c = space.take((size_t)splits * q.M * q.ldc * sizeof(float));
        q.c_type = CCDC_F32;
        joins.j[joins.count++] = {static_cast<const float *>(q.c), c, q.M, q.N, q.ldc, ldc, splits, c_type};
    }
    void run_products(const MmaProduct *q, int count, MmaEpilogue e, MmaTile tile) {
        if (rc != CCDC_OK) return;
        rc = mma_launch(q, count, e, type(), tile, sms, s);
    }
    void run_joins() {
        if (!joins.count || rc != CCDC_OK) return;
        long long most = 0;
        for (int i = 0; i < joins.count; ++i) most = std::max(most, joins.j[i].rows * (joins.j[i].cols / 4 + 1));
        rc = launch_small(k_ffn_join, joins, most, joins.count, sms, s);
    }

    void forward(const void *x, long long ldx, const void *wg, const void *wu, long long ldw, const void *wd, long long ldd,
                 void *y, long long ldy, char *saved) {
        float *h = reinterpret_cast<float *>(saved), *u = saved ? reinterpret_cast<float *>(saved + wide_bytes(M, F)) : nullptr;
        char *kept = saved ? saved + 2 * wide_bytes(M, F) : nullptr;
        if (M <= rows_most(dtype)) {        // few rows: bound by the weights' bytes, not by products
            void *a = kept ? kept : space.take((size_t)M * pitch(F) * type_bytes(dtype));
            if (!fits()) return;
            RowsProduct p = {M, F, D, x, wg, wu, ldx, ldw, a, pitch(F), h, u, act, dtype, false};
            rc = rows_launch(p, sms, s);
            if (rc != CCDC_OK) return;
            RowsProduct q = {M, D, F, a, wd, nullptr, pitch(F), ldd, y, ldy, nullptr, nullptr, act, dtype, true};
            rc = rows_launch(q, sms, s);
            return;
        }
        const MmaMatrix X = operand(x, M, D, ldx), G = operand(wg, F, D, ldw), U = operand(wu, F, D, ldw);
        const MmaMatrix W = operand(wd, D, F, ldd);
        void *a = kept ? kept : space.take(inner_bytes(M, F, dtype));
        MmaProduct p = {};
        p.M = M, p.N = F, p.K = D, p.terms = 1, p.act = act;
        p.a[0] = {X, false}, p.b[0] = {G, false}, p.b[1] = {U, false};
        p.h = h, p.u = u;
        p.out[0] = inner(a);
        Shape first = {M, F, steps_of(D, 1), 1};
        const MmaTile tile = choose_tiles(&first, 1, MMA_GATE, dtype == CCDC_F32, sms);
        MmaProduct q = {};
        q.M = M, q.N = D, q.K = F, q.terms = 1, q.a[0] = {inner(a), false}, q.b[0] = {W, false};
        Shape second = {M, D, steps_of(F, 1), 1};
        const MmaTile tile2 = choose_tiles(&second, 1, MMA_STORE, dtype == CCDC_F32, sms);
        to_output(q, second.splits, y, ldy, dtype);
        if (!fits()) return;
        run_copies();
        run_products(&p, 1, MMA_GATE, tile);
        run_products(&q, 1, MMA_STORE, tile2);
        run_joins();
    }

    // binary32, few rows
    void few_backward(const void *dy, long long lddy, const void *x, long long ldx, const void *wg, const void *wu,
                      long long ldw, const void *wd, long long ldd, char *saved, void *dx, long long lddx, void *dwg, void *dwu,
                      void *dwd) {
        auto f = [](const void *p) { return static_cast<const float *>(p); };
        const float *a = f(saved + 2 * wide_bytes(M, F));
        const long long ld = pitch(F), ldo = pitch(D);
        float *dh = static_cast<float *>(space.take((size_t)M * ld * 4)), *du = static_cast<float *>(space.take((size_t)M * ld * 4));
        const int cuts = few_across_splits(M, F, D, 1, sms), cuts_x = few_across_splits(M, D, F, 2, sms);
        float *da = static_cast<float *>(space.take((size_t)cuts * M * ld * 4));
        float *parts = static_cast<float *>(space.take((size_t)cuts_x * M * ldo * 4));
        if (!fits()) return;
        rc = few_across({M, F, D, 1, cuts, {f(dy), nullptr}, {f(wd), nullptr}, lddy, ldd, ld, da}, s);
        if (rc == CCDC_OK)
            rc = few_gate_back({M, F, ld, cuts, act, da, reinterpret_cast<float *>(saved),
                                reinterpret_cast<float *>(saved + wide_bytes(M, F)), dh, du}, s);
        if (rc == CCDC_OK && dx) {
            rc = few_across({M, D, F, 2, cuts_x, {dh, du}, {f(wg), f(wu)}, ld, ldw, ldo, parts}, s);
            joins.j[joins.count++] = {parts, dx, M, D, ldo, lddx, cuts_x, CCDC_F32};
            run_joins();
        }
        FewOuters o = {};
        o.M = M;
        if (dwg) o.o[o.count++] = {dh, f(x), ld, ldx, F, D, static_cast<float *>(dwg)};
        if (dwu) o.o[o.count++] = {du, f(x), ld, ldx, F, D, static_cast<float *>(dwu)};
        if (dwd) o.o[o.count++] = {f(dy), a, lddy, ld, D, F, static_cast<float *>(dwd)};
        if (rc == CCDC_OK && o.count) rc = few_outer(o, s);
    }

    void backward(const void *dy, long long lddy, const void *x, long long ldx, const void *wg, const void *wu, long long ldw,
                  const void *wd, long long ldd, char *saved, void *dx, long long lddx, void *dwg, void *dwu, void *dwd,
                  int grad_dtype) {
        if (dtype == CCDC_F32 && M <= FEW_MOST) {
            few_backward(dy, lddy, x, ldx, wg, wu, ldw, wd, ldd, saved, dx, lddx, dwg, dwu, dwd);
            return;
        }
        const MmaMatrix DY = operand(dy, M, D, lddy), X = operand(x, M, D, ldx), G = operand(wg, F, D, ldw);
        const MmaMatrix U = operand(wu, F, D, ldw), W = operand(wd, D, F, ldd);
        const MmaMatrix A = inner(saved + 2 * wide_bytes(M, F));
        const MmaMatrix DH = inner(space.take(inner_bytes(M, F, dtype))), DU = inner(space.take(inner_bytes(M, F, dtype)));
        MmaProduct p = {};
        p.M = M, p.N = F, p.K = D, p.terms = 1, p.act = act;
        p.a[0] = {DY, false}, p.b[0] = {W, true};
        p.h = reinterpret_cast<float *>(saved), p.u = reinterpret_cast<float *>(saved + wide_bytes(M, F));
        p.out[0] = DH, p.out[1] = DU;
        Shape first = {M, F, steps_of(D, 1), 1};
        const MmaTile tile = choose_tiles(&first, 1, MMA_GATE_BACK, dtype == CCDC_F32, sms);
        MmaProduct q[4] = {};
        Shape shapes[4];
        void *to[4];
        int n = 0;
        auto add = [&](long long m, long long nn, long long k, int terms, void *c) {
            q[n].M = m, q[n].N = nn, q[n].K = k, q[n].terms = terms;
            shapes[n] = {m, nn, steps_of(k, terms), 1};
            to[n] = c;
            return &q[n++];
        };
        MmaProduct *r = add(M, D, F, 2, dx);        // the longest items first
        r->a[0] = {DH, false}, r->b[0] = {G, true}, r->a[1] = {DU, false}, r->b[1] = {U, true};
        r = add(F, D, M, 1, dwg);
        r->a[0] = {DH, true}, r->b[0] = {X, true};
        r = add(F, D, M, 1, dwu);
        r->a[0] = {DU, true}, r->b[0] = {X, true};
        r = add(D, F, M, 1, dwd);
        r->a[0] = {DY, true}, r->b[0] = {A, true};
        // tiles and cuts are those of the whole set, so that leaving an output out changes no other output's bits
        const MmaTile tile2 = choose_tiles(shapes, n, MMA_STORE, dtype == CCDC_F32, sms);
        int wanted = 0;
        for (int i = 0; i < n; ++i) {
            if (!to[i] && !plan_only) continue;
            const bool is_dx = q[i].terms == 2;
            to_output(q[i], shapes[i].splits, to[i], is_dx ? lddx : q[i].N, is_dx ? dtype : grad_dtype);
            q[wanted++] = q[i];
        }
        n = wanted;
        if (!fits()) return;
        run_copies();
        run_products(&p, 1, MMA_GATE_BACK, tile);
        run_products(q, n, MMA_STORE, tile2);
        run_joins();
    }
};

// The most that a call of these sizes can need: with everything wanted.
size_t forward_bytes(long long M, long long D, long long F, int dtype, bool aligned, int sms) {
    Call c = {M, D, F, dtype, 0, sms, true, aligned};
    c.forward(nullptr, D, nullptr, nullptr, D, nullptr, F, nullptr, D, nullptr);
    return c.space.used + 256;
}
size_t backward_bytes(long long M, long long D, long long F, int dtype, bool aligned, int sms) {
    Call c = {M, D, F, dtype, 0, sms, true, aligned};
    c.backward(nullptr, D, nullptr, D, nullptr, nullptr, D, nullptr, F, nullptr, nullptr, D, nullptr, nullptr, nullptr, dtype);
    return c.space.used + 256;
}

}  // namespace

extern "C" {

size_t ccdc_ffn_saved_bytes(long long M, long long F, int dtype) {
    if (check_ffn(M, 1, F, dtype, 0) != CCDC_OK) return 0;
    return 2 * wide_bytes(M, F) + inner_bytes(M, F, dtype);
}

size_t ccdc_ffn_workspace_bytes(long long M, long long D, long long F, int dtype, int backward, int aligned) {
    if (check_ffn(M, D, F, dtype, 0) != CCDC_OK) return 0;
    if (M == 0) return 256;
    int rc;
    int sms = block_sm_count(&rc);
    if (rc != CCDC_OK) sms = 148;
    return backward ? backward_bytes(M, D, F, dtype, aligned != 0, sms) : forward_bytes(M, D, F, dtype, aligned != 0, sms);
}

int ccdc_ffn_forward(long long M, long long D, long long F, int dtype, int act, const void *x, long long ldx,
                     const void *w_gate, const void *w_up, long long ldw, const void *w_down, long long ldd, void *y,
                     long long ldy, void *saved, void *workspace, size_t workspace_bytes, void *stream) {
    int rc = check_ffn(M, D, F, dtype, act);
    if (rc != CCDC_OK) return rc;
    if (M == 0) return CCDC_OK;
    if (!x || !w_gate || !w_up || !w_down || !y || !workspace || ldx < D || ldw < D || ldd < F || ldy < D ||
        !aligned_to(saved, 16) || !aligned_to(workspace, 16))
        return CCDC_EINVAL;
    if (workspace_bytes < 256) return CCDC_ESIZE;
    Call c = {M, D, F, dtype, act, 0, false, false};
    c.sms = block_sm_count(&rc);
    if (rc != CCDC_OK) return rc;
    c.space.base = static_cast<char *>(workspace), c.space.size = workspace_bytes;
    c.s = static_cast<cudaStream_t>(stream);
    c.forward(x, ldx, w_gate, w_up, ldw, w_down, ldd, y, ldy, static_cast<char *>(saved));
    return c.rc;
}

int ccdc_ffn_backward(long long M, long long D, long long F, int dtype, int grad_dtype, int act, const void *dy,
                      long long lddy, const void *x, long long ldx, const void *w_gate, const void *w_up, long long ldw,
                      const void *w_down, long long ldd, const void *saved, void *dx, long long lddx, void *dw_gate,
                      void *dw_up, void *dw_down, void *workspace, size_t workspace_bytes, void *stream) {
    int rc = check_ffn(M, D, F, dtype, act);
    if (rc != CCDC_OK) return rc;
    if (grad_dtype != dtype && grad_dtype != CCDC_F32) return CCDC_EINVAL;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (M == 0) {
        for (void *g : {dw_gate, dw_up, dw_down})
            if (g) {
                const cudaError_t e = cudaMemsetAsync(g, 0, (size_t)D * F * type_bytes(grad_dtype), s);
                if (e != cudaSuccess) return ccdc_internal_cuda_fail((int)e);
            }
        return CCDC_OK;
    }
    if (!dy || !x || !w_gate || !w_up || !w_down || !saved || !workspace || lddy < D || ldx < D || ldw < D || ldd < F ||
        (dx && lddx < D) || !aligned_to(saved, 16) || !aligned_to(workspace, 16))
        return CCDC_EINVAL;
    if (workspace_bytes < 256) return CCDC_ESIZE;
    Call c = {M, D, F, dtype, act, 0, false, false};
    c.sms = block_sm_count(&rc);
    if (rc != CCDC_OK) return rc;
    c.space.base = static_cast<char *>(workspace), c.space.size = workspace_bytes;
    c.s = s;
    char *keep = static_cast<char *>(const_cast<void *>(saved));
    c.backward(dy, lddy, x, ldx, w_gate, w_up, ldw, w_down, ldd, keep, dx, lddx, dw_gate, dw_up, dw_down, grad_dtype);
    return c.rc;
}

int ccdc_block_status(void) {
    int failed = 0;
    const int rc = mma_status(&failed);
    return rc != CCDC_OK ? rc : failed ? CCDC_ESTATE : CCDC_OK;
}

}  // extern "C"
