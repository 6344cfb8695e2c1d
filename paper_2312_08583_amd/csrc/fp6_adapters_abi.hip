// C ABI of the operators around the frozen layer (include/fp6_linear.h): argument checks and dispatch.  Everything here runs on the host;
// no device allocation, no synchronisation, and no C++ exception leaves it.
#include "../../include/fp6_linear.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <vector>

#include "fp6_adamw.hpp"
#include "fp6_internal.hpp"

namespace fp6 {

static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

static bool shape_ok(int64_t N, int64_t K)
{
    return N > 0 && K > 0 && N % FP6_TILE == 0 && K % FP6_TILE == 0 && N <= (int64_t)1 << 30 && K <= (int64_t)1 << 30 &&
           N * K <= (int64_t)1 << 40;
}

static bool rows_ok(int64_t M) { return M > 0 && M <= (int64_t)1 << 24; }

// A range of device memory.
struct Span {
    const void* p;
    size_t bytes;
};

static bool overlap(Span a, Span b)
{
    if (!a.p || !b.p || !a.bytes || !b.bytes) return false;
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return x < y + b.bytes && y < x + a.bytes;
}

static int lora_numbers(int type, int64_t rank, int64_t adapters)
{
    if (type != FP6_F16 && type != FP6_BF16) return FP6_ERR_VALUE;
    if (rank < 8 || rank > FP6_LORA_RANK_MAX || rank % 8 || adapters < 1 || adapters > 65535) return FP6_ERR_VALUE;
    return FP6_OK;
}

// The threads of a launch are counted in 32 bits, its workgroups of 256 in 24: half of them for each of the steps that share a launch.  (Up to
// 512 rows workgroups take at least 16 rows and 256 columns, adapters may be dealt to 16 of them; above, with so many, 1024 rows and 64 columns.)
static bool lora_fits(int64_t M, int64_t columns, int64_t adapters)
{
    const int64_t few = (M + 15) / 16 * ((columns + 255) / 256) * std::min<int64_t>(adapters, 16), many = (M + 1023) / 1024 * ((columns + 63) / 64);
    return (M <= 512 ? few : many) < (int64_t)1 << 22;
}
static bool backward_fits(int64_t M, int64_t N, int64_t K, int64_t adapters)
{
    return lora_fits(M, std::max(N, K), adapters) && (std::max(N, K) + 127) / 128 * adapters < (int64_t)1 << 23;
}

static int lora_check(int type, int64_t M, const fp6_lora_problem* pr, int count, int64_t adapters)
{
    if (!pr) return FP6_ERR_NULL;
    if (count < 1 || count > FP6_GROUP_MAX || !rows_ok(M)) return FP6_ERR_SHAPE;
    int64_t columns = 0;
    for (int i = 0; i < count; i++) {
        const int bad = lora_numbers(type, pr[i].rank, adapters);
        if (bad != FP6_OK) return bad;
        if (!shape_ok(pr[i].N, pr[i].K)) return FP6_ERR_SHAPE;
        columns += pr[i].N;
    }
    return lora_fits(M, columns, adapters) ? FP6_OK : FP6_ERR_SHAPE;
}

static int lora_any(int type, int64_t M, const fp6_lora_problem* pr, int count, int64_t adapters, const int32_t* index,
                    const float* scaling, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!pr) return FP6_ERR_NULL;
    for (int i = 0; i < count && i < FP6_GROUP_MAX; i++)
        if (!pr[i].X || !pr[i].A || !pr[i].B || !pr[i].Y || !pr[i].out) return FP6_ERR_NULL;
    const int bad = lora_check(type, M, pr, count, adapters);
    if (bad != FP6_OK) return bad;
    for (int i = 0; i < count; i++)
        if (!aligned16(pr[i].X) || !aligned16(pr[i].A) || !aligned16(pr[i].B) || !aligned16(pr[i].Y) || !aligned16(pr[i].out) ||
            !aligned16(pr[i].hidden))
            return FP6_ERR_ALIGN;
    if (!aligned16(index) || !aligned16(scaling) || !aligned16(workspace)) return FP6_ERR_ALIGN;
    const size_t need = lora_workspace(M, pr, count, (int)adapters);
    if (!workspace || workspace_bytes < need) return FP6_ERR_WORKSPACE;
    const Span common[] = {{index, (size_t)M * 4}, {scaling, (size_t)adapters * 4}, {workspace, need}};
    for (int i = 0; i < count; i++) {
        const Span written[] = {{pr[i].out, (size_t)(M * pr[i].N) * 2}, {pr[i].hidden, (size_t)(M * pr[i].rank) * 4}};
        if (overlap(written[0], written[1])) return FP6_ERR_OVERLAP;
        for (const Span& w : written) {
            for (const Span& c : common)
                if (overlap(w, c)) return FP6_ERR_OVERLAP;
            for (int k = 0; k < count; k++) {
                const Span read[] = {{pr[k].X, (size_t)(M * pr[k].K) * 2}, {pr[k].A, (size_t)(adapters * pr[k].rank * pr[k].K) * 2},
                                     {pr[k].B, (size_t)(adapters * pr[k].rank * pr[k].N) * 2}, {pr[k].Y, (size_t)(M * pr[k].N) * 2}};
                for (int r = 0; r < 4; r++)
                    if (overlap(w, read[r]) && !(r == 3 && k == i && w.p == read[3].p && w.p == pr[i].out)) return FP6_ERR_OVERLAP;
                if (k != i && (overlap(w, Span{pr[k].out, (size_t)(M * pr[k].N) * 2}) ||
                               overlap(w, Span{pr[k].hidden, (size_t)(M * pr[k].rank) * 4})))
                    return FP6_ERR_OVERLAP;
            }
        }
        const Span read[] = {{pr[i].X, (size_t)(M * pr[i].K) * 2}, {pr[i].A, (size_t)(adapters * pr[i].rank * pr[i].K) * 2},
                             {pr[i].B, (size_t)(adapters * pr[i].rank * pr[i].N) * 2}, {pr[i].Y, (size_t)(M * pr[i].N) * 2}, common[0], common[1]};
        for (const Span& r : read)
            if (overlap(r, common[2])) return FP6_ERR_OVERLAP;
    }
    (void)hipGetLastError();      // (an earlier call's)
    return launch_lora(type == FP6_BF16, M, pr, count, (int)adapters, index, scaling, workspace, (hipStream_t)stream) == hipSuccess
               ? FP6_OK
               : FP6_ERR_HIP;
}

static bool grad_format(int format)
{
    return format == kE3M2 || format == kE3M1 || format == kE3M2H || format == kE3M2B;
}

// The layer that computes the gradient has N inputs and K outputs.  Its workspace lies at the start, dY * ratio behind it.
static size_t grad_inner(int format, int64_t M, int64_t N, int64_t K)
{
    const size_t need = format == kE3M2   ? fp6_linear_workspace_bytes(M, K, N)
                        : format == kE3M1 ? fp5_linear_workspace_bytes(M, K, N, 0, 0)
                                          : fp6_linear_v2_workspace_bytes(M, K, N, 0, 0);
    return std::max(need, kZeroBytes);
}

static bool is_number(double v, double lo, double hi) { return v >= lo && v < hi; }

struct PlanLayout {
    int64_t item, items;
    size_t bytes;
};

static bool plan_layout(const fp6_adamw_tensor* t, int64_t count, PlanLayout* l)
{
    if (!t || count < 1 || count > (int64_t)1 << 24) return false;
    int64_t elements = 0;
    for (int64_t i = 0; i < count; i++) {
        if (t[i].count < 0 || t[i].count > (int64_t)1 << 40) return false;
        elements += t[i].count;
        if (elements > (int64_t)1 << 41) return false;
    }
    l->item = adamw_item(elements);
    l->items = 0;
    for (int64_t i = 0; i < count; i++) l->items += (t[i].count + l->item - 1) / l->item;
    l->bytes = sizeof(AdamwHeader) + (size_t)l->items * sizeof(AdamwItem);
    return true;
}

static bool adamw_types(int state_bits, int grad_type, int copy_type)
{
    return (state_bits == 8 || state_bits == 32) && (grad_type == FP6_F16 || grad_type == FP6_BF16 || grad_type == FP6_F32) &&
           (copy_type == FP6_F16 || copy_type == FP6_BF16 || copy_type == FP6_NO_COPY);
}

static int adamw_plan(const fp6_adamw_tensor* t, int64_t count, int state_bits, int grad_type, int copy_type, void* plan_host,
                      size_t plan_bytes, int64_t* items)
{
    if (!t || !plan_host || !items) return FP6_ERR_NULL;
    PlanLayout l;
    if (!adamw_types(state_bits, grad_type, copy_type)) return FP6_ERR_VALUE;
    if (!plan_layout(t, count, &l)) return FP6_ERR_VALUE;
    if (plan_bytes < l.bytes) return FP6_ERR_WORKSPACE;
    struct Range {
        uintptr_t begin, end;
        bool written;
    };
    std::vector<Range> ranges;
    ranges.reserve((size_t)count * 7);
    for (int64_t i = 0; i < count; i++) {
        const fp6_adamw_tensor& x = t[i];
        if (x.count == 0) continue;
        if (!x.param || !x.grad || !x.first || !x.second) return FP6_ERR_NULL;
        if (state_bits == 8 && (!x.first_scales || !x.second_scales)) return FP6_ERR_NULL;
        if (copy_type != FP6_NO_COPY && !x.copy) return FP6_ERR_NULL;
        if (!aligned16(x.param) || !aligned16(x.grad) || !aligned16(x.first) || !aligned16(x.second) ||
            (copy_type != FP6_NO_COPY && !aligned16(x.copy)))
            return FP6_ERR_ALIGN;
        const size_t n = (size_t)x.count, state = state_bits == 8 ? 1 : 4, blocks = (n + 255) / 256;
        auto add = [&](const void* p, size_t bytes, bool written) { ranges.push_back(Range{(uintptr_t)p, (uintptr_t)p + bytes, written}); };
        add(x.param, 4 * n, true);
        add(x.grad, grad_type == FP6_F32 ? 4 * n : 2 * n, false);
        add(x.first, state * n, true);
        add(x.second, state * n, true);
        if (state_bits == 8) {
            add(x.first_scales, blocks, true);
            add(x.second_scales, blocks, true);
        }
        if (copy_type != FP6_NO_COPY) add(x.copy, 2 * n, true);
    }
    std::sort(ranges.begin(), ranges.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
    // the furthest end of what lies before, written or not
    uintptr_t end_written = 0, end_any = 0;
    for (const Range& r : ranges) {
        if (r.begin < end_written || (r.written && r.begin < end_any)) return FP6_ERR_OVERLAP;
        end_any = std::max(end_any, r.end);
        if (r.written) end_written = std::max(end_written, r.end);
    }
    unsigned char* at = (unsigned char*)plan_host;
    AdamwHeader h{};
    h.magic = kAdamwMagic;
    h.kind = adamw_kind(state_bits, grad_type, copy_type);
    h.items = (uint64_t)l.items;
    std::memcpy(at, &h, sizeof h);
    at += sizeof h;
    const int64_t grad_bytes = grad_type == FP6_F32 ? 4 : 2, state = state_bits == 8 ? 1 : 4;
    uint32_t id = 0;                     // (numbers of elements wrap at 2^32: they only feed a hash)
    for (int64_t i = 0; i < count; i++) {
        const fp6_adamw_tensor& x = t[i];
        for (int64_t e = 0; e < x.count; e += l.item, at += sizeof(AdamwItem)) {
            AdamwItem item{x.param + e, (const char*)x.grad + grad_bytes * e, (char*)x.first + state * e, (char*)x.second + state * e,
                           nullptr, nullptr, nullptr, id + (uint32_t)e, (uint32_t)std::min(l.item, x.count - e)};
            if (state_bits == 8) {
                item.first_scales = x.first_scales + e / 256;
                item.second_scales = x.second_scales + e / 256;
            }
            if (copy_type != FP6_NO_COPY) item.copy = x.copy + e;
            std::memcpy(at, &item, sizeof item);
        }
        id += (uint32_t)((x.count + 255) / 256) * 256u;
    }
    *items = l.items;
    return FP6_OK;
}

}  // namespace fp6

using namespace fp6;

extern "C" {

size_t fp6_lora_group_workspace_bytes(int64_t M, const fp6_lora_problem* problems, int count, int64_t adapters)
{
    return lora_check(FP6_F16, M, problems, count, adapters) == FP6_OK ? lora_workspace(M, problems, count, (int)adapters) : 0;
}

size_t fp6_lora_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t rank, int64_t adapters)
{
    fp6_lora_problem p{};
    p.N = N;
    p.K = K;
    p.rank = rank;
    return fp6_lora_group_workspace_bytes(M, &p, 1, adapters);
}

int fp6_lora_group(int type, int64_t M, const fp6_lora_problem* problems, int count, int64_t adapters, const int32_t* index,
                   const float* scaling, void* workspace, size_t workspace_bytes, void* stream)
{
    return lora_any(type, M, problems, count, adapters, index, scaling, workspace, workspace_bytes, stream);
}

int fp6_lora(int type, const uint16_t* X, int64_t M, const uint16_t* A, const uint16_t* B, int64_t adapters, int64_t rank,
             const int32_t* index, const float* scaling, const uint16_t* Y, int64_t N, int64_t K, uint16_t* out, float* hidden,
             void* workspace, size_t workspace_bytes, void* stream)
{
    const fp6_lora_problem p{X, A, B, Y, out, hidden, N, K, rank};
    return lora_any(type, M, &p, 1, adapters, index, scaling, workspace, workspace_bytes, stream);
}

size_t fp6_lora_backward_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t rank, int64_t adapters)
{
    if (!rows_ok(M) || !shape_ok(N, K) || lora_numbers(FP6_F16, rank, adapters) != FP6_OK || !backward_fits(M, N, K, adapters)) return 0;
    return lora_backward_workspace(M, N, K, (int)rank, (int)adapters);
}

int fp6_lora_backward(int type, const uint16_t* dY, const uint16_t* X, const float* hidden, int64_t M, const uint16_t* A,
                      const uint16_t* B, int64_t adapters, int64_t rank, const int32_t* index, const float* scaling,
                      const uint16_t* dX, uint16_t* out, float* dA, float* dB, int accumulate, int64_t N, int64_t K,
                      void* workspace, size_t workspace_bytes, void* stream)
{
    if (!dY || !X || !hidden || !A || !B || !dA || !dB || !dX != !out) return FP6_ERR_NULL;
    const int bad = lora_numbers(type, rank, adapters);
    if (bad != FP6_OK) return bad;
    if (!rows_ok(M) || !shape_ok(N, K) || !backward_fits(M, N, K, adapters)) return FP6_ERR_SHAPE;
    const void* all[] = {dY, X, hidden, A, B, index, scaling, dX, out, dA, dB, workspace};
    for (const void* p : all)
        if (!aligned16(p)) return FP6_ERR_ALIGN;
    const size_t need = lora_backward_workspace(M, N, K, (int)rank, (int)adapters);
    if (!workspace || workspace_bytes < need) return FP6_ERR_WORKSPACE;
    const size_t a = (size_t)(adapters * rank * K), b = (size_t)(adapters * rank * N);
    const Span written[] = {{out, (size_t)(M * K) * 2}, {dA, a * 4}, {dB, b * 4}, {workspace, need}};
    const Span read[] = {{dY, (size_t)(M * N) * 2}, {X, (size_t)(M * K) * 2}, {hidden, (size_t)(M * rank) * 4}, {A, a * 2}, {B, b * 2},
                         {index, (size_t)M * 4}, {scaling, (size_t)adapters * 4}, {dX, (size_t)(M * K) * 2}};
    for (int w = 0; w < 4; w++) {
        for (int r = 0; r < 8; r++)
            if (overlap(written[w], read[r]) && !(w == 0 && r == 7 && out == dX)) return FP6_ERR_OVERLAP;
        for (int v = 0; v < w; v++)
            if (overlap(written[w], written[v])) return FP6_ERR_OVERLAP;
    }
    const LoraBackward g{dY, X, hidden, A, B, index, scaling, dX, out, dA, dB, M, N, K, (int)rank, (int)adapters, accumulate != 0};
    (void)hipGetLastError();
    return launch_lora_backward(type == FP6_BF16, g, workspace, (hipStream_t)stream) == hipSuccess ? FP6_OK : FP6_ERR_HIP;
}

int fp6_transpose_pack(int format, const void* hi_plane, const void* lo_plane, const uint16_t* scales, int64_t N, int64_t K,
                       void* hi_t, void* lo_t, uint16_t* scales_t, float* ratio, void* stream)
{
    if (!hi_plane || !lo_plane || !scales || !hi_t || !lo_t || !scales_t || !ratio) return FP6_ERR_NULL;
    if (!grad_format(format)) return FP6_ERR_VARIANT;
    if (!shape_ok(N, K)) return FP6_ERR_SHAPE;
    const void* all[] = {hi_plane, lo_plane, scales, hi_t, lo_t, scales_t, ratio};
    for (const void* p : all)
        if (!aligned16(p)) return FP6_ERR_ALIGN;
    const size_t hi = (size_t)(N * K / 2), lo = (size_t)(N * K / (format == kE3M1 ? 8 : 4));
    const Span written[] = {{hi_t, hi}, {lo_t, lo}, {scales_t, (size_t)K * 2}, {ratio, (size_t)N * 4}};
    const Span read[] = {{hi_plane, hi}, {lo_plane, lo}, {scales, (size_t)N * 2}};
    for (int w = 0; w < 4; w++) {
        for (const Span& r : read)
            if (overlap(written[w], r)) return FP6_ERR_OVERLAP;
        for (int v = 0; v < w; v++)
            if (overlap(written[w], written[v])) return FP6_ERR_OVERLAP;
    }
    (void)hipGetLastError();
    return launch_transpose_pack(format, hi_plane, lo_plane, scales, N, K, hi_t, lo_t, scales_t, ratio, (hipStream_t)stream) == hipSuccess
               ? FP6_OK
               : FP6_ERR_HIP;
}

size_t fp6_linear_grad_workspace_bytes(int format, int64_t M, int64_t N, int64_t K)
{
    if (!grad_format(format) || !rows_ok(M) || !shape_ok(N, K)) return 0;
    return grad_inner(format, M, N, K) + (size_t)(M * N) * 2;
}

int fp6_linear_grad(int format, const uint16_t* dY, int64_t M, const void* hi_t, const void* lo_t, const uint16_t* scales_t,
                    const float* ratio, int64_t N, int64_t K, uint16_t* dX, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!dY || !hi_t || !lo_t || !scales_t || !ratio || !dX) return FP6_ERR_NULL;
    if (!grad_format(format)) return FP6_ERR_VARIANT;
    if (!rows_ok(M) || !shape_ok(N, K)) return FP6_ERR_SHAPE;
    const void* all[] = {dY, hi_t, lo_t, scales_t, ratio, dX, workspace};
    for (const void* p : all)
        if (!aligned16(p)) return FP6_ERR_ALIGN;
    const size_t inner = grad_inner(format, M, N, K), need = inner + (size_t)(M * N) * 2;
    if (!workspace || workspace_bytes < need) return FP6_ERR_WORKSPACE;
    const Span written[] = {{dX, (size_t)(M * K) * 2}, {workspace, need}};
    const Span read[] = {{dY, (size_t)(M * N) * 2}, {hi_t, (size_t)(N * K / 2)}, {lo_t, (size_t)(N * K / (format == kE3M1 ? 8 : 4))},
                         {scales_t, (size_t)K * 2}, {ratio, (size_t)N * 4}};
    for (const Span& w : written)
        for (const Span& r : read)
            if (overlap(w, r)) return FP6_ERR_OVERLAP;
    if (overlap(written[0], written[1])) return FP6_ERR_OVERLAP;
    uint16_t* scaled = (uint16_t*)((unsigned char*)workspace + inner);
    (void)hipGetLastError();
    if (launch_scale_rows(format == kE3M2B, dY, ratio, M, N, scaled, (hipStream_t)stream) != hipSuccess) return FP6_ERR_HIP;
    if (format == kE3M2) return fp6_linear(scaled, M, hi_t, lo_t, scales_t, K, N, dX, workspace, inner, stream);
    if (format == kE3M1) return fp5_linear(scaled, M, hi_t, lo_t, scales_t, K, N, dX, workspace, inner, stream, 0, 0);
    return format == kE3M2H ? fp6_linear_v2(scaled, M, hi_t, lo_t, scales_t, K, N, dX, workspace, inner, stream, 0, 0)
                            : fp6_linear_v2_bf16(scaled, M, hi_t, lo_t, scales_t, K, N, dX, workspace, inner, stream, 0, 0);
}

size_t fp6_adamw_plan_bytes(const fp6_adamw_tensor* tensors, int64_t count)
{
    PlanLayout l;
    return plan_layout(tensors, count, &l) ? l.bytes : 0;
}

int fp6_adamw_plan(const fp6_adamw_tensor* tensors, int64_t count, int state_bits, int grad_type, int copy_type, void* plan_host,
                   size_t plan_bytes, int64_t* items)
{
    try {
        return adamw_plan(tensors, count, state_bits, grad_type, copy_type, plan_host, plan_bytes, items);
    } catch (...) {          // no host memory for the list of ranges
        return FP6_ERR_WORKSPACE;
    }
}

int fp6_adamw(void* plan, int64_t items, int state_bits, int grad_type, int copy_type, int32_t* step,
              const fp6_adamw_options* options, void* stream)
{
    if (!plan || !step || !options) return FP6_ERR_NULL;
    if (!adamw_types(state_bits, grad_type, copy_type) || items < 0 || items > (int64_t)1 << 31) return FP6_ERR_VALUE;
    const fp6_adamw_options& o = *options;
    if (!is_number(o.beta1, 0, 1) || !is_number(o.beta2, 0, 1) || !is_number(o.eps, 0, INFINITY) || !is_number(o.weight_decay, 0, INFINITY) ||
        (!o.lr_device && !is_number(o.lr, 0, INFINITY)))
        return FP6_ERR_VALUE;
    const void* scalars[] = {step, o.lr_device, o.grad_scale, o.found_inf};
    for (const void* p : scalars)
        if ((uintptr_t)p & 3) return FP6_ERR_ALIGN;
    if (!aligned16(plan)) return FP6_ERR_ALIGN;
    const AdamwCall call{o.lr, o.beta1, o.beta2, o.eps, o.weight_decay, o.lr_device, o.grad_scale, o.found_inf, o.seed};
    (void)hipGetLastError();
    // (no element at all: one workgroup counts the step on)
    return launch_adamw(state_bits, grad_type, copy_type, (AdamwHeader*)plan, items, step, call, (hipStream_t)stream) == hipSuccess
               ? FP6_OK
               : FP6_ERR_HIP;
}

}  // extern "C"
