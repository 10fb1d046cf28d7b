// Rotary positions: the handle that holds the frequencies, and the rotation of a tensor of rows (or, transposed, of its gradient).
#include <cmath>
#include <new>

#include "rope_rows.h"
#include "rows_apart.h"

namespace veda {

struct RopeApply {
    RopeArgs rope;
    const char* x;
    char* y;
    int64_t sx_b, sx_h, sx_n, sy_b, sy_h, sy_n;   // bytes
    const int32_t* positions;
    int64_t pos_b;
    int32_t heads, tokens, head_dim, units, log_tb, hb;
    RowOrder order;
};

template <typename E, bool kChunks> __global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeApply a) {
    extern __shared__ float2 cs[];
    const int tb = 1 << a.log_tb, t0 = blockIdx.x << a.log_tb, n = min(tb, a.tokens - t0);
    const int h0 = blockIdx.y * a.hb, nh = min(a.hb, a.heads - h0);
    const int64_t b = blockIdx.z;
    const int32_t* pos = a.positions + b * a.pos_b + (int64_t)t0 * a.rope.axes;
    rope_angles(a.rope, n, [&](int t, int axis) { return pos[t * a.rope.axes + axis]; }, cs);
    __syncthreads();
    const char* x = a.x + b * a.sx_b + t0 * a.sx_n;
    char* y = a.y + b * a.sy_b + t0 * a.sy_n;
    const RowAt at(a.order, a.log_tb, nh);
    rope_rows<E, kChunks>(a.rope, a.head_dim, a.units, at.rows(n), cs,
                          [&](int r) {
                              int t, h;
                              at.find(r, t, h);
                              h += h0;
                              RowMove m{x + h * a.sx_h + t * a.sx_n, y + h * a.sy_h + t * a.sy_n, t, true};
                              if (t >= n) m.dst = nullptr;
                              return m;
                          });
}

}  // namespace veda

using veda::aligned16;

extern "C" veda_status veda_rope_create(const veda_rope_config* c, veda_rope** out) {
    if (!c || !out) return VEDA_ERR_INVALID_ARG;
    if (c->axes < 1 || c->axes > 3 || c->head_dim < 1) return VEDA_ERR_INVALID_ARG;
    if (c->pairs != VEDA_ROPE_INTERLEAVED && c->pairs != VEDA_ROPE_HALVES) return VEDA_ERR_INVALID_ARG;
    const bool ntk = c->scaling == VEDA_ROPE_NTK, parts = c->scaling == VEDA_ROPE_BY_PARTS;
    if (c->scaling != VEDA_ROPE_PLAIN && c->scaling != VEDA_ROPE_LINEAR && !ntk && !parts) return VEDA_ERR_INVALID_ARG;
    if (!(c->base > 1.0) || !std::isfinite(c->base) || !(c->amplitude >= 0.0) || !std::isfinite(c->amplitude)) return VEDA_ERR_INVALID_ARG;
    const double factor = c->scaling == VEDA_ROPE_PLAIN ? 1.0 : c->factor;
    if (!(factor >= 1.0) || !std::isfinite(factor)) return VEDA_ERR_INVALID_ARG;
    if (parts && (!(c->trained_len > 0.0) || !std::isfinite(c->trained_len) || !(c->beta_slow >= 0.0) || !(c->beta_fast > c->beta_slow) ||
                  !std::isfinite(c->beta_fast)))
        return VEDA_ERR_INVALID_ARG;
    int64_t rot = 0;
    for (int a = 0; a < c->axes; ++a) {
        if (c->axis_dim[a] < 2 || c->axis_dim[a] % 2 || (ntk && c->axis_dim[a] == 2)) return VEDA_ERR_INVALID_ARG;
        rot += c->axis_dim[a];
    }
    if (rot > c->head_dim) return VEDA_ERR_INVALID_ARG;
    if (c->head_dim % 8 || c->head_dim > 512) return VEDA_ERR_UNSUPPORTED;
    veda_rope* r = new (std::nothrow) veda_rope();
    if (!r) return veda::hip_fail(hipErrorOutOfMemory, "veda_rope_create");
    const double two_pi = 6.283185307179586476925286766559;
    hipError_t e = hipErrorOutOfMemory;
    try {
        r->cfg = *c;
        r->rot = (int32_t)rot;
        r->amplitude = c->amplitude > 0.0 ? c->amplitude : parts ? 0.1 * std::log(factor) + 1.0 : 1.0;
        for (int a = 0; a < c->axes; ++a) {
            const double w = c->axis_dim[a], base = ntk ? c->base * std::pow(factor, w / (w - 2.0)) : c->base;
            for (int i = 0; i < c->axis_dim[a] / 2; ++i) {
                double f = std::pow(base, -2.0 * i / w);
                if (c->scaling == VEDA_ROPE_LINEAR) f /= factor;
                if (parts) {
                    const double g = (c->trained_len * f / two_pi - c->beta_slow) / (c->beta_fast - c->beta_slow);
                    const double keep = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
                    f *= keep + (1.0 - keep) / factor;
                }
                r->freq.push_back(f);
            }
        }
        std::vector<double> turns(r->freq);
        for (double& f : turns) f /= two_pi;
        e = hipGetDevice(&r->device);
        if (e == hipSuccess) e = hipMalloc((void**)&r->d_turns, turns.size() * sizeof(double));
        if (e == hipSuccess) e = hipMemcpy(r->d_turns, turns.data(), turns.size() * sizeof(double), hipMemcpyHostToDevice);
    } catch (const std::exception&) {
        e = hipErrorOutOfMemory;
    }
    if (e != hipSuccess) {
        veda_status st = veda::hip_fail(e, "veda_rope_create");
        veda_rope_destroy(r);
        return st;
    }
    *out = r;
    return VEDA_OK;
}

extern "C" void veda_rope_destroy(veda_rope* r) {
    if (!r) return;
    if (r->d_turns) (void)hipFree(r->d_turns);
    delete r;
}

extern "C" veda_status veda_rope_frequencies(const veda_rope* r, double* freq, double* amplitude) {
    if (!r) return VEDA_ERR_INVALID_ARG;
    if (freq)
        for (size_t i = 0; i < r->freq.size(); ++i) freq[i] = r->freq[i];
    if (amplitude) *amplitude = r->amplitude;
    return VEDA_OK;
}

extern "C" veda_status veda_rope_apply(const veda_rope* rope, veda_dtype dtype, int32_t batch, int32_t heads, int32_t tokens,
                                       const void* x, veda_strides sx, const int32_t* positions, int64_t position_stride,
                                       int32_t transpose, void* y, veda_strides sy, void* stream) {
    if (!rope || batch < 0 || heads < 0 || tokens < 0 || (transpose != 0 && transpose != 1)) return VEDA_ERR_INVALID_ARG;
    if (dtype != VEDA_F32 && dtype != VEDA_BF16) return VEDA_ERR_INVALID_ARG;
    if (batch == 0 || heads == 0 || tokens == 0) return VEDA_OK;
    if (!x || !y || !positions) return VEDA_ERR_INVALID_ARG;
    const int d = rope->cfg.head_dim, es = dtype == VEDA_BF16 ? 2 : 4;
    if (position_stride < 0 || (position_stride > 0 && position_stride < (int64_t)tokens * rope->cfg.axes)) return VEDA_ERR_INVALID_ARG;
    // an axis of one entry has no stride, whatever it is given as
    if (batch == 1) sx.b = sy.b = 0;
    if (heads == 1) sx.h = sy.h = 0;
    if (tokens == 1) sx.n = sy.n = 0;
    if (sx.b < 0 || sx.h < 0 || sx.n < 0 || sy.b < 0 || sy.h < 0 || sy.n < 0) return VEDA_ERR_INVALID_ARG;
    const veda::RowsApart apart = veda::rows_apart({tokens, sy.n}, {heads, sy.h}, {batch, sy.b}, d);
    if (apart != veda::RowsApart::kApart) return apart == veda::RowsApart::kShare ? VEDA_ERR_INVALID_ARG : VEDA_ERR_UNSUPPORTED;
    if (x == y && (sx.n != sy.n || sx.h != sy.h || sx.b != sy.b)) return VEDA_ERR_INVALID_ARG;
    if (!aligned16(x) || !aligned16(y) || (sx.b * es) % 16 || (sx.h * es) % 16 || (sx.n * es) % 16 || (sy.b * es) % 16 ||
        (sy.h * es) % 16 || (sy.n * es) % 16)
        return VEDA_ERR_UNSUPPORTED;
    int device = -1;
    VEDA_HIP_TRY(hipGetDevice(&device));
    if (device != rope->device) return VEDA_ERR_INVALID_ARG;
    veda::RopeApply a;
    a.rope = veda::rope_args(rope, transpose);
    a.x = (const char*)x; a.y = (char*)y;
    a.sx_b = sx.b * es; a.sx_h = sx.h * es; a.sx_n = sx.n * es;
    a.sy_b = sy.b * es; a.sy_h = sy.h * es; a.sy_n = sy.n * es;
    a.positions = positions; a.pos_b = position_stride;
    a.heads = heads; a.tokens = tokens; a.head_dim = d;
    const int chunk = 16 / es;
    const bool chunks = veda::rope_in_chunks(a.rope, chunk);
    a.units = veda::rope_units(a.rope, d, chunk, chunks);
    a.rope.through = veda::rope_whole_lines(a.rope, d, es);
    veda::rope_blocks(tokens, batch, heads, &a.log_tb, &a.hb);
    a.order = veda::row_order(sx.h < sx.n);
    const int64_t head_groups = ((int64_t)heads + a.hb - 1) / a.hb;
    const int64_t gx = ((int64_t)tokens + (1 << a.log_tb) - 1) >> a.log_tb;
    if (gx >= 1 << 24 || head_groups > 65535 || batch > 65535) return VEDA_ERR_UNSUPPORTED;   // a grid has less than 2^32 threads
    const dim3 grid((unsigned)gx, (unsigned)head_groups, (unsigned)batch);
    const size_t lds = (size_t)a.rope.half * sizeof(float2) << a.log_tb;
    const hipStream_t s = (hipStream_t)stream;
    if (dtype == VEDA_BF16 && chunks) hipLaunchKernelGGL((veda::rope_kernel<uint16_t, true>), grid, dim3(veda::kRopeThreads), lds, s, a);
    else if (dtype == VEDA_BF16) hipLaunchKernelGGL((veda::rope_kernel<uint16_t, false>), grid, dim3(veda::kRopeThreads), lds, s, a);
    else if (chunks) hipLaunchKernelGGL((veda::rope_kernel<uint32_t, true>), grid, dim3(veda::kRopeThreads), lds, s, a);
    else hipLaunchKernelGGL((veda::rope_kernel<uint32_t, false>), grid, dim3(veda::kRopeThreads), lds, s, a);
    return veda::launch_status("veda_rope_apply");
}
