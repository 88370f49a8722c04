// The binding's side of the steps over microscaled pages and shared prefixes: the same checks of the arguments and the same calls of the C
// entries as binding.py makes for the other steps, compiled.  A server makes these calls once per layer and token, and in Python
// the checks of ten to fifteen tensors and the marshalling of up to 39 arguments take longer than the kernels of a step of a few tokens
// (8 tokens appended and their rows read back: 22 us bound by the host, 9 us so).
//
// Host code only.  Nothing here synchronises or allocates, but for a step's workspace where the caller gave none.
#include <torch/extension.h>

#include <c10/core/impl/VirtualGuardImpl.h>

#include <cstdint>

#include "../../include/snapkv.h"

namespace {

typedef c10::optional<at::Tensor> maybe;

[[noreturn]] void refuse(const std::string& what) { throw py::value_error(what); }
#define REQUIRE(cond, what) \
    do {                    \
        if (!(cond)) refuse(what); \
    } while (0)

int dtype_code(const at::Tensor& t) {
    switch (t.scalar_type()) {
        case at::kBFloat16: return SNAPKV_DTYPE_BF16;
        case at::kFloat: return SNAPKV_DTYPE_F32;
        case at::kHalf: return SNAPKV_DTYPE_F16;
        default: refuse("q/k/v must be bfloat16, float16 or float32");
    }
}

// The device of a call's tensors.  Calls run on the current device, on a stream of it: no other is taken.
struct Call {
    c10::Device device;
    Call(const at::Tensor& t, const char* name) : device(t.device()) {
        REQUIRE(t.is_cuda(), std::string(name) + " must be a GPU tensor");
        const auto current = c10::impl::VirtualGuardImpl(device.type()).getDevice();
        REQUIRE(device.index() == current.index(), std::string(name) + " is on cuda:" + std::to_string(device.index()) +
                                                       ", the current device is cuda:" + std::to_string(current.index()));
    }
    void check(const at::Tensor& t, const char* name, at::ScalarType type, bool contiguous) const {
        REQUIRE(t.is_cuda(), std::string(name) + " must be a GPU tensor");
        REQUIRE(t.device() == device, std::string(name) + " is on cuda:" + std::to_string(t.device().index()) + ", other tensors of the call on cuda:" +
                                          std::to_string(device.index()));
        REQUIRE(t.scalar_type() == type, std::string(name) + " must be " + c10::toString(type) + ", got " + c10::toString(t.scalar_type()));
        REQUIRE(contiguous, std::string(name) + " must be contiguous (its rows, where strides are allowed)");
    }
    // Address of a contiguous tensor of this type on this device.
    void* at(const at::Tensor& t, const char* name, at::ScalarType type) const {
        check(t, name, type, t.is_contiguous());
        return t.data_ptr();
    }
    void* at(const maybe& t, const char* name, at::ScalarType type) const { return t ? at(*t, name, type) : nullptr; }
};
template <typename T> const int32_t* ints(T* p) { return static_cast<const int32_t*>(p); }

// Address and (row, head) strides of a [T, H, D] view with contiguous rows; the stride of a dimension of one does not matter.
struct Rows {
    void* p = nullptr;
    int64_t row = 0, head = 0;
    Rows() = default;
    Rows(const Call& call, const at::Tensor& t, const char* name, at::ScalarType type) {
        call.check(t, name, type, t.stride(2) == 1);
        p = t.data_ptr();
        row = t.size(0) > 1 ? t.stride(0) : t.size(2);
        head = t.size(1) > 1 ? t.stride(1) : 0;
    }
};

int narrow(int64_t n) {
    REQUIRE(n <= INT32_MAX, "a dimension of a tensor is beyond 2^31");
    return (int)n;
}

bool is(const at::Tensor& t, std::initializer_list<int64_t> shape) { return t.sizes() == at::IntArrayRef(shape); }

// Which codes microscaled pages hold, by their width.
int cache_of(const at::Tensor& kp, const at::Tensor& ks, const at::Tensor& vp, const at::Tensor& vs, int64_t Hkv, int64_t D) {
    const bool fits = kp.dim() == 4 && vp.sizes() == kp.sizes() && kp.size(2) == Hkv && (kp.size(3) == D || kp.size(3) == D / 2) &&
                      is(ks, {kp.size(0), kp.size(1), Hkv, D / 32}) && vs.sizes() == ks.sizes();
    REQUIRE(fits, "microscaled pages must be codes [num_pages, page_size, Hkv, D] or [.., D / 2] and scales [.., D / 32]");
    return kp.size(3) == D ? SNAPKV_CACHE_FP8 : SNAPKV_CACHE_FP4;
}

// Workspace of a step: the caller's, or one for this call.
struct Workspace {
    at::Tensor owner;
    void* p = nullptr;
    size_t bytes = 0;
    template <typename F> Workspace(const Call& call, const maybe& given, F need) {
        if (given) {
            p = call.at(*given, "workspace", at::kByte);
            bytes = (size_t)given->numel();
        } else if ((bytes = need()) > 0) {
            owner = at::empty({(int64_t)bytes}, at::TensorOptions().dtype(at::kByte).device(call.device));
            p = owner.data_ptr();
        }
    }
};

void* stream_of(int64_t s) { return reinterpret_cast<void*>(s); }

int append_paged_mx(const at::Tensor& k, const at::Tensor& v, const at::Tensor& kp, const at::Tensor& ks, const at::Tensor& vp,
                    const at::Tensor& vs, const at::Tensor& table, const at::Tensor& starts, const maybe& cu, const maybe& positions,
                    const maybe& cos, const maybe& sin, bool interleaved, const maybe& q, const maybe& q_out, const maybe& k_out,
                    int64_t stream) {
    REQUIRE(k.dim() == 3 && v.sizes() == k.sizes(), "k and v must both be [T, Hkv, D]");
    const int64_t T = k.size(0), Hkv = k.size(1), D = k.size(2);
    const int cache = cache_of(kp, ks, vp, vs, Hkv, D);
    REQUIRE(table.dim() == 2, "block_table must be [B, columns]");
    const int64_t B = table.size(0);
    REQUIRE(is(starts, {B}), "starts must be [B]");
    REQUIRE(!cu || is(*cu, {B + 1}), "cu_seqlens must be [B + 1]");
    REQUIRE(!positions || is(*positions, {T}), "positions must be [T]");
    REQUIRE(cos.has_value() == sin.has_value() && (!cos || (cos->dim() == 2 && sin->sizes() == cos->sizes())),
            "cos and sin must both be [positions, rot_dim / 2]");
    REQUIRE(q.has_value() == q_out.has_value() && (!q || (q->dim() == 3 && q->size(0) == T && q->size(2) == D && q_out->sizes() == q->sizes())),
            "q and q_out must both be [T, Hq, D]");
    REQUIRE(!k_out || k_out->sizes() == k.sizes(), "k_out must be [T, Hkv, D]");
    const Call call(k, "k");
    const auto type = k.scalar_type();
    const int64_t Hq = q ? q->size(1) : 0;
    const Rows rk(call, k, "k", type), rv(call, v, "v", type);
    const Rows rq = Hq ? Rows(call, *q, "q", type) : Rows(), ro = Hq ? Rows(call, *q_out, "q_out", type) : Rows();
    const Rows rc = k_out ? Rows(call, *k_out, "k_out", type) : Rows();
    return snapkv_append_paged_mx(
        dtype_code(k), cache, rq.p, rk.p, rv.p, ints(call.at(cu, "cu_seqlens", at::kInt)), ints(call.at(starts, "starts", at::kInt)),
        ints(call.at(positions, "positions", at::kInt)), T, narrow(B), narrow(Hq), narrow(Hkv), narrow(D), rq.row, rq.head, rk.row, rk.head, rv.row, rv.head,
        static_cast<const float*>(call.at(cos, "cos", at::kFloat)), static_cast<const float*>(call.at(sin, "sin", at::kFloat)),
        cos ? cos->size(0) : 0, cos ? narrow(2 * cos->size(1)) : 0, interleaved ? 1 : 0, call.at(kp, "k_pages", at::kByte),
        call.at(ks, "k_scales", at::kByte), call.at(vp, "v_pages", at::kByte), call.at(vs, "v_scales", at::kByte),
        ints(call.at(table, "block_table", at::kInt)), table.size(1), kp.size(0), narrow(kp.size(1)), ro.p, ro.row, ro.head, rc.p, rc.row, rc.head,
        stream_of(stream));
}

int read_paged_mx(const at::Tensor& kp, const at::Tensor& ks, const at::Tensor& vp, const at::Tensor& vs, const at::Tensor& table,
                  const at::Tensor& starts, const at::Tensor& k_out, const at::Tensor& v_out, const maybe& cu, int64_t stream) {
    REQUIRE(k_out.dim() == 3 && v_out.sizes() == k_out.sizes() && v_out.scalar_type() == k_out.scalar_type(), "k_out and v_out disagree on their shapes or types");
    const int64_t T = k_out.size(0), Hkv = k_out.size(1), D = k_out.size(2);
    const int cache = cache_of(kp, ks, vp, vs, Hkv, D);
    REQUIRE(table.dim() == 2, "block_table must be [B, columns]");
    const int64_t B = table.size(0);
    REQUIRE(is(starts, {B}) && (!cu || is(*cu, {B + 1})), "starts must be [B] and cu_seqlens [B + 1]");
    const Call call(k_out, "k_out");
    const Rows rk(call, k_out, "k_out", k_out.scalar_type()), rv(call, v_out, "v_out", k_out.scalar_type());
    return snapkv_read_paged_mx(dtype_code(k_out), cache, call.at(kp, "k_pages", at::kByte), call.at(ks, "k_scales", at::kByte),
                                call.at(vp, "v_pages", at::kByte), call.at(vs, "v_scales", at::kByte),
                                ints(call.at(table, "block_table", at::kInt)), table.size(1), kp.size(0), narrow(kp.size(1)),
                                ints(call.at(cu, "cu_seqlens", at::kInt)), ints(call.at(starts, "starts", at::kInt)), T, narrow(B), narrow(Hkv), narrow(D),
                                rk.p, rk.row, rk.head, rv.p, rv.row, rv.head, stream_of(stream));
}

// q, out [B, Hq, D], out_lse [B, Hq], block_table [B, columns], lens [B]
void check_step(const at::Tensor& q, const at::Tensor& table, const at::Tensor& lens, const at::Tensor& out, const maybe& lse) {
    REQUIRE(q.dim() == 3, "q must be [B, Hq, D]");
    const int64_t B = q.size(0);
    REQUIRE(table.dim() == 2 && table.size(0) == B && is(lens, {B}), "block_table must be [B, columns] and lens [B]");
    REQUIRE(out.sizes() == q.sizes() && (!lse || is(*lse, {B, q.size(1)})), "out must be [B, Hq, D] and out_lse [B, Hq]");
}

int decode_attention_paged_mx(const at::Tensor& q, const at::Tensor& kp, const at::Tensor& ks, const at::Tensor& vp, const at::Tensor& vs,
                              const at::Tensor& table, const at::Tensor& lens, int64_t max_len, const at::Tensor& out, const maybe& lse,
                              const maybe& workspace, int64_t stream) {
    check_step(q, table, lens, out, lse);
    REQUIRE(kp.dim() == 4, "k_pages must be [num_pages, page_size, Hkv, D] or [.., D / 2]");
    const int B = narrow(q.size(0)), Hq = narrow(q.size(1)), D = narrow(q.size(2)), Hkv = narrow(kp.size(2));
    const int cache = cache_of(kp, ks, vp, vs, Hkv, D);
    const Call call(q, "q");
    const Workspace ws(call, workspace, [&] { return snapkv_decode_paged_mx_workspace_bytes(B, Hq, Hkv, D, max_len); });
    return snapkv_decode_attention_paged_mx(
        dtype_code(q), cache, call.at(q, "q", q.scalar_type()), call.at(kp, "k_pages", at::kByte), call.at(ks, "k_scales", at::kByte),
        call.at(vp, "v_pages", at::kByte), call.at(vs, "v_scales", at::kByte), ints(call.at(table, "block_table", at::kInt)), table.size(1),
        kp.size(0), narrow(kp.size(1)), ints(call.at(lens, "lens", at::kInt)), max_len, B, Hq, Hkv, D, call.at(out, "out", q.scalar_type()),
        static_cast<float*>(call.at(lse, "out_lse", at::kFloat)), ws.p, ws.bytes, stream_of(stream));
}

int decode_attention_shared(const at::Tensor& q, const at::Tensor& kp, const at::Tensor& vp, const at::Tensor& prefix_table,
                            const at::Tensor& prefix_lens, int64_t max_prefix, const at::Tensor& table, const at::Tensor& lens, int64_t max_len,
                            const at::Tensor& out, const maybe& lse, const maybe& cu, const maybe& ks, const maybe& vs, const maybe& workspace,
                            int64_t stream) {
    check_step(q, table, lens, out, lse);
    REQUIRE(kp.dim() == 4, "k_pages must be [num_pages, page_size, Hkv, D], or of codes [.., D / 2]");
    const int B = narrow(q.size(0)), Hq = narrow(q.size(1)), D = narrow(q.size(2)), Hkv = narrow(kp.size(2));
    REQUIRE(ks.has_value() == vs.has_value(), "k_scales and v_scales must both be given");
    const int cache = ks ? cache_of(kp, *ks, vp, *vs, Hkv, D) : SNAPKV_CACHE_PLAIN;
    REQUIRE(ks || (kp.size(3) == D && vp.sizes() == kp.sizes()), "q, k_pages and v_pages disagree on their shapes");
    REQUIRE(prefix_table.dim() == 2, "prefix_table must be [G, columns]");
    const int64_t G = prefix_table.size(0);
    REQUIRE(is(prefix_lens, {G}) && (cu ? is(*cu, {G + 1}) : G == 1), "prefix_lens must be [G] and cu_groups [G + 1] (None: one group)");
    const Call call(q, "q");
    const auto type = ks ? at::kByte : q.scalar_type();
    const Workspace ws(call, workspace, [&] { return snapkv_decode_shared_workspace_bytes(B, narrow(G), Hq, Hkv, D, max_prefix, max_len); });
    return snapkv_decode_attention_shared(
        dtype_code(q), cache, call.at(q, "q", q.scalar_type()), call.at(kp, "k_pages", type), call.at(ks, "k_scales", at::kByte),
        call.at(vp, "v_pages", type), call.at(vs, "v_scales", at::kByte), kp.size(0), narrow(kp.size(1)), ints(call.at(cu, "cu_groups", at::kInt)),
        narrow(G), ints(call.at(prefix_table, "prefix_table", at::kInt)), prefix_table.size(1), ints(call.at(prefix_lens, "prefix_lens", at::kInt)),
        max_prefix, ints(call.at(table, "block_table", at::kInt)), table.size(1), ints(call.at(lens, "lens", at::kInt)), max_len, B, Hq, Hkv, D,
        call.at(out, "out", q.scalar_type()), static_cast<float*>(call.at(lse, "out_lse", at::kFloat)), ws.p, ws.bytes, stream_of(stream));
}

}  // namespace

PYBIND11_MODULE(_steps, m) {
    m.def("append_paged_mx", &append_paged_mx);
    m.def("read_paged_mx", &read_paged_mx);
    m.def("decode_attention_paged_mx", &decode_attention_paged_mx);
    m.def("decode_attention_shared", &decode_attention_shared);
}
