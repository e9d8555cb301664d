// Python side of the serving operators: torch tensors to the argument structs of bcast_serve.h.
//
// A call's tensors are checked against each other here (types, shapes, device, contiguous innermost dimension)
// and described to the C entry point, which checks the rest; nothing is computed.  Native because a decode step's
// kernels take about as long as marshalling a dozen tensors in Python does (33 us of 44 us measured).
// Every function returns (code, outputs or what was wrong, whether the stream is being captured into a graph).
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGraphsC10Utils.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/utils/pybind.h>

#include <initializer_list>
#include <optional>
#include <string>
#include <vector>

#include "bcast_serve.h"

namespace py = pybind11;
using at::Tensor;
using Maybe = std::optional<Tensor>;

namespace {

struct Refused {
    std::string why;
};

void need(bool ok, const char *why)
{
    if (!ok) throw Refused{why};
}

int dtype_of(const Tensor &t, bool with_fp32)
{
    switch (t.scalar_type()) {
    case at::kBFloat16: return BCAST_SERVE_BF16;
    case at::kHalf: return BCAST_SERVE_FP16;
    case at::kFloat:
        if (with_fp32) return BCAST_SERVE_FP32;
    default: throw Refused{std::string("type ") + c10::toString(t.scalar_type())};
    }
}

std::string list(at::IntArrayRef v)
{
    std::string s = "(";
    for (size_t i = 0; i < v.size(); i++) s += (i ? ", " : "") + std::to_string(v[i]);
    return s + ")";
}

// One tensor against what the call expects of it.
void expect(const Tensor &t, const char *name, at::ScalarType type, at::IntArrayRef shape, const at::Device &dev)
{
    const bool inner = shape.empty() || shape.back() <= 1 || (t.dim() > 0 && t.stride(-1) == 1);
    if (t.scalar_type() == type && t.sizes() == shape && t.device() == dev && inner) return;
    throw Refused{std::string(name) + ": " + list(t.sizes()) + " " + c10::toString(t.scalar_type()) + " on " + t.device().str() +
                  " with strides " + list(t.strides()) + ", expected " + list(shape) + " " + c10::toString(type) + " on " + dev.str() +
                  ", last dimension contiguous"};
}

// Strides of the first `n` dimensions; where a dimension has one entry its stride means nothing and is given
// as that of a contiguous array, rounded up to 8.
void strides(const Tensor &t, int n, int64_t *out)
{
    int64_t run = 1;
    for (int64_t i = t.dim() - 1; i >= 0; i--) {
        const int64_t s = t.size(i) == 1 ? run : t.stride(i);
        run = std::max(run, (s * t.size(i) + 7) / 8 * 8);
        if (i < n) out[i] = s;
    }
}

const Tensor *given(const Maybe &t) { return t ? &*t : nullptr; }
const void *pointer(const Maybe &t) { return t ? t->data_ptr() : nullptr; }

// Where a call runs: the device of its tensors, the stream that was named (-1: torch's current one) and the
// workspace, which lives on stream `ws_of` for torch's allocator.
struct Place {
    c10::cuda::CUDAGuard device;
    c10::cuda::CUDAStream stream;
    std::optional<c10::cuda::CUDAStreamGuard> guard;

    Place(const Tensor &t, int64_t raw) : device(check(t)), stream(c10::cuda::getCurrentCUDAStream(t.get_device()))
    {
        if (raw < 0 || (int64_t)stream.stream() == raw) return;
        stream = raw ? c10::cuda::getStreamFromExternal((cudaStream_t)raw, (c10::DeviceIndex)t.get_device())
                     : c10::cuda::getDefaultCUDAStream((c10::DeviceIndex)t.get_device());
        guard.emplace(stream);
    }
    // On a stream that was named, torch does not know of the tensors' use: their memory is not to be handed out again
    // before this stream is done with it, should the caller let go of them.
    void use(std::initializer_list<const Tensor *> tensors) const
    {
        if (!guard) return;
        for (const Tensor *t : tensors)
            if (t) c10::cuda::CUDACachingAllocator::recordStream(t->storage().data_ptr(), stream);
    }
    static at::Device check(const Tensor &t)
    {
        need(t.is_cuda(), "tensors on a CUDA device");
        return t.device();
    }
    template <typename Args>
    void use(Args &a, const Maybe &ws, int64_t ws_of) const
    {
        a.workspace = ws ? ws->data_ptr() : nullptr;
        a.workspace_bytes = ws ? (uint64_t)ws->nbytes() : 0;
        if (ws && ws_of != (int64_t)stream.stream()) c10::cuda::CUDACachingAllocator::recordStream(ws->storage().data_ptr(), stream);
    }
};

Tensor output(const Maybe &out, const char *name, at::IntArrayRef shape, at::ScalarType type, const at::Device &dev)
{
    if (!out) return at::empty(shape, at::TensorOptions().dtype(type).device(dev));
    expect(*out, name, type, shape, dev);
    return *out;
}

// The call itself; BCAST_ERR_CAPACITY comes back with the bytes that are needed.
template <typename Args>
py::tuple finish(int (*call)(const Args *, void *), int64_t (*size)(const Args *), const Args &a, const Place &place, py::object outputs)
{
    int64_t bytes = size(&a);
    int code = bytes < 0 ? (int)bytes : (uint64_t)bytes > a.workspace_bytes ? BCAST_ERR_CAPACITY : call(&a, place.stream.stream());
    if (code == BCAST_ERR_CAPACITY) return py::make_tuple(code, bytes, false);
    if (code) return py::make_tuple(code, "", false);
    // (asked of the stream of `place`, which is the current one here)
    return py::make_tuple(code, std::move(outputs), c10::cuda::currentStreamCaptureStatusMayInitCtx() != c10::cuda::CaptureStatus::None);
}

template <typename F>
py::tuple guarded(F f)
{
    try {
        return f();
    } catch (const Refused &r) {
        return py::make_tuple((int)BCAST_ERR_INVAL, r.why, false);
    }
}

py::tuple linear(const Tensor &x, const Tensor &weight, const Maybe &bias, const Maybe &lora_a, const Maybe &lora_b, const Maybe &adapter,
                 const Maybe &scale, const Maybe &out, const Maybe &ws, int64_t ws_of, int64_t raw)
{
    return guarded([&] {
        need(x.dim() == 2 && weight.dim() == 2, "x and weight have two dimensions");
        bcast_serve_linear_args a = {};
        a.dtype = dtype_of(x, false);
        const auto type = x.scalar_type();
        const at::Device dev = x.device();
        a.tokens = x.size(0);
        a.k = x.size(1);
        a.n = weight.size(0);
        expect(x, "x", type, x.sizes(), dev);
        expect(weight, "weight", type, {a.n, a.k}, dev);
        if (bias) expect(*bias, "bias", type, {a.n}, dev);
        need(lora_a.has_value() == lora_b.has_value() && lora_a.has_value() == adapter.has_value() && lora_a.has_value() == scale.has_value(),
             "lora_a, lora_b, adapter and scale go together");
        if (lora_a) {
            need(lora_a->dim() == 3, "lora_a has three dimensions");
            const int64_t L = lora_a->size(0), R = lora_a->size(1);
            need(L < (1 << 30) && R < (1 << 30), "lora_a is too large");
            expect(*lora_a, "lora_a", type, {L, R, a.k}, dev);
            expect(*lora_b, "lora_b", type, {L, a.n, R}, dev);
            expect(*adapter, "adapter", at::kInt, {a.tokens}, dev);
            expect(*scale, "scale", at::kFloat, {L}, dev);
            a.num_adapters = (int32_t)L;
            a.rank = (int32_t)R;
            strides(*lora_a, 2, a.lora_a_stride);
            strides(*lora_b, 2, a.lora_b_stride);
        }
        const Place place(x, raw);
        place.use({&x, &weight, given(bias), given(lora_a), given(lora_b), given(adapter), given(scale), given(out)});
        const Tensor y = output(out, "out", {a.tokens, a.n}, type, dev);
        a.x = x.data_ptr();
        a.weight = weight.data_ptr();
        a.bias = pointer(bias);
        a.lora_a = pointer(lora_a);
        a.lora_b = pointer(lora_b);
        a.adapter = (const int32_t *)pointer(adapter);
        a.scale = (const float *)pointer(scale);
        a.y = y.data_ptr();
        strides(x, 1, &a.x_stride);
        strides(weight, 1, &a.weight_stride);
        strides(y, 1, &a.y_stride);
        place.use(a, ws, ws_of);
        return finish(bcast_serve_linear, bcast_serve_linear_workspace, a, place, py::cast(y));
    });
}

py::tuple attn(const Tensor &q, const Tensor &prefix_k, const Tensor &prefix_v, const Tensor &own_k, const Tensor &own_v, const Tensor &own_len,
               const Maybe &page_table, std::optional<double> scale, const Maybe &out, const Maybe &lse, const Maybe &ws, int64_t ws_of, int64_t raw)
{
    return guarded([&] {
        need(q.dim() == 4 && prefix_k.dim() == 3 && own_k.dim() == 4, "q and own_k have four dimensions, prefix_k three");
        bcast_serve_attn_args a = {};
        a.dtype = dtype_of(q, false);
        const auto type = q.scalar_type();
        const at::Device dev = q.device();
        const int64_t B = q.size(0), n = q.size(1), HQ = q.size(2), D = q.size(3), P = prefix_k.size(0), H = prefix_k.size(1);
        need(std::max({B, n, HQ, D, H}) < (1 << 30), "q is too large");
        expect(q, "q", type, q.sizes(), dev);
        expect(prefix_k, "prefix_k", type, {P, H, D}, dev);
        expect(prefix_v, "prefix_v", type, {P, H, D}, dev);
        const int64_t own = page_table ? own_k.size(0) : B, each = own_k.size(1);
        expect(own_k, "own_k", type, {own, each, H, D}, dev);
        expect(own_v, "own_v", type, {own, each, H, D}, dev);
        expect(own_len, "own_len", at::kInt, {B}, dev);
        a.own_cap = each;
        if (page_table) {
            need(page_table->dim() == 2 && each >= 1 && each < (1 << 30), "page_table has two dimensions, a page at least one token");
            expect(*page_table, "page_table", at::kInt, {B, page_table->size(1)}, dev);
            a.page_size = (int32_t)each;
            a.num_pages = own;
            a.own_cap = each * page_table->size(1);
            strides(*page_table, 1, &a.page_table_stride);
        }
        if (lse) {
            expect(*lse, "lse", at::kFloat, {B, n, HQ}, dev);
            need(lse->is_contiguous(), "lse is contiguous");
        }
        const Place place(q, raw);
        place.use({&q, &prefix_k, &prefix_v, &own_k, &own_v, &own_len, given(page_table), given(out), given(lse)});
        const Tensor o = output(out, "out", {B, n, HQ, D}, type, dev);
        a.batch = (int32_t)B;
        a.new_tokens = (int32_t)n;
        a.q_heads = (int32_t)HQ;
        a.kv_heads = (int32_t)H;
        a.dim = (int32_t)D;
        a.scale = scale ? (float)*scale : D > 0 ? (float)(1.0 / std::sqrt((double)D)) : 0.0f;
        a.prefix_len = P;
        a.q = q.data_ptr();
        a.prefix_k = prefix_k.data_ptr();
        a.prefix_v = prefix_v.data_ptr();
        a.own_k = own_k.data_ptr();
        a.own_v = own_v.data_ptr();
        a.own_len = (const int32_t *)own_len.data_ptr();
        a.page_table = (const int32_t *)pointer(page_table);
        a.out = o.data_ptr();
        a.lse = (float *)pointer(lse);
        strides(q, 3, a.q_stride);
        strides(o, 3, a.out_stride);
        strides(prefix_k, 2, a.prefix_k_stride);
        strides(prefix_v, 2, a.prefix_v_stride);
        strides(own_k, 3, a.own_k_stride);
        strides(own_v, 3, a.own_v_stride);
        place.use(a, ws, ws_of);
        return finish(bcast_serve_attn, bcast_serve_attn_workspace, a, place, py::cast(o));
    });
}

py::tuple verify(const Tensor &logits, const Tensor &draft_probs, const Tensor &draft_tokens, const Tensor &uniforms, const Tensor &noise,
                 const Tensor &temperature, const Maybe &accepted, const Maybe &tokens, const Maybe &ws, int64_t ws_of, int64_t raw)
{
    return guarded([&] {
        need(logits.dim() == 3 && logits.size(1) >= 1, "logits has three dimensions and at least one row");
        bcast_serve_verify_args a = {};
        a.dtype = dtype_of(logits, true);
        const at::Device dev = logits.device();
        const int64_t B = logits.size(0), n = logits.size(1) - 1, V = logits.size(2);
        need(B < (1 << 30) && n < (1 << 30), "logits is too large");
        expect(logits, "logits", logits.scalar_type(), logits.sizes(), dev);
        expect(draft_probs, "draft_probs", at::kFloat, {B, n, V}, dev);
        expect(draft_tokens, "draft_tokens", at::kInt, {B, n}, dev);
        expect(uniforms, "uniforms", at::kFloat, {B, n}, dev);
        need(draft_tokens.is_contiguous() && uniforms.is_contiguous(), "draft_tokens and uniforms are contiguous");
        expect(noise, "noise", at::kFloat, {B, V}, dev);
        expect(temperature, "temperature", at::kFloat, {B}, dev);
        const Place place(logits, raw);
        place.use({&logits, &draft_probs, &draft_tokens, &uniforms, &noise, &temperature, given(accepted), given(tokens)});
        const Tensor c = output(accepted, "accepted", {B}, at::kInt, dev), t = output(tokens, "tokens", {B, n + 1}, at::kInt, dev);
        need(t.is_contiguous(), "tokens is contiguous");
        a.batch = (int32_t)B;
        a.drafts = (int32_t)n;
        a.vocab = V;
        a.logits = logits.data_ptr();
        a.draft_probs = (const float *)draft_probs.data_ptr();
        a.uniforms = (const float *)uniforms.data_ptr();
        a.noise = (const float *)noise.data_ptr();
        a.temperature = (const float *)temperature.data_ptr();
        a.draft_tokens = (const int32_t *)draft_tokens.data_ptr();
        a.accepted = (int32_t *)c.data_ptr();
        a.tokens = (int32_t *)t.data_ptr();
        strides(logits, 2, a.logits_stride);
        strides(draft_probs, 2, a.draft_probs_stride);
        strides(noise, 1, &a.noise_stride);
        place.use(a, ws, ws_of);
        return finish(bcast_serve_verify, bcast_serve_verify_workspace, a, place, py::make_tuple(c, t));
    });
}

}  // namespace

PYBIND11_MODULE(_serve_native, m)
{
    m.def("linear", &linear);
    m.def("attn", &attn);
    m.def("verify", &verify);
    m.def("strides", [](const Tensor &t, int n) {
        std::vector<int64_t> s((size_t)std::max(n, 0));
        strides(t, n, s.data());
        return py::tuple(py::cast(s));
    });
}
