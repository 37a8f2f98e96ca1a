// train_binding.cpp -- the training-step entry points as torch sees them: the
// common form of each call (outputs allocated here, on the current stream)
// marshalled in C++, since for short calls the Python marshalling costs several
// times the kernels.  Checks, results and errors are those of train.py, which
// takes every other form of a call itself.  Every step of the computation runs
// behind the C ABI of include/iso.h, as everywhere.
#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/utils/pybind.h>

#include <string>

#include "iso.h"

namespace py = pybind11;

namespace {

[[noreturn]] void value_error(const std::string& s) { throw py::value_error(s); }
[[noreturn]] void type_error(const std::string& s) { throw py::type_error(s); }

int32_t code_of(at::ScalarType t, const char* name) {
    if (t == at::kBFloat16) return ISO_BF16;
    if (t == at::kFloat) return ISO_F32;
    type_error(std::string(name) + " must be bfloat16 or float32, got " + c10::toString(t));
}

iso_mat mat(const at::Tensor& t, const char* name) {
    if (t.dim() != 2) value_error(std::string(name) + " must be a 2-D tensor");
    const int32_t code = code_of(t.scalar_type(), name);
    if (!t.is_cuda()) value_error(std::string(name) + " must be a CUDA tensor");
    const int64_t rows = t.size(0), cols = t.size(1);
    int64_t ld = t.stride(0);
    if (t.stride(1) != 1 && cols > 1) value_error(std::string(name) + " must have unit stride along its rows");
    if (ld < cols) {
        if (rows > 1 && cols) value_error(std::string(name) + " has overlapping rows");
        ld = cols;
    }
    return {t.data_ptr(), rows, cols, ld, code, 0};
}

at::Tensor empty(int64_t rows, int64_t cols, at::ScalarType t, const at::Tensor& like) {
    return at::empty({rows, cols}, like.options().dtype(t));
}
iso_mat new_mat(const at::Tensor& t) {
    return {t.data_ptr(), t.size(0), t.size(1), t.size(1), t.scalar_type() == at::kBFloat16 ? ISO_BF16 : ISO_F32, 0};
}

void* stream_of(const at::Tensor& first) {
    const auto index = first.get_device();
    if (index != c10::cuda::current_device())
        value_error("tensors are on cuda:" + std::to_string((int)index) + ", the current device is cuda:" +
                    std::to_string((int)c10::cuda::current_device()));
    return c10::cuda::getCurrentCUDAStream(index).stream();
}
void same_device(const at::Tensor& a, const at::Tensor& b) {
    if (a.device() != b.device())
        value_error("tensors on different devices: " + a.device().str() + " and " + b.device().str());
}

at::Tensor scratch(size_t bytes, const at::Tensor& like) {
    return at::empty({(int64_t)bytes + 256}, like.options().dtype(at::kByte));
}
void* aligned(const at::Tensor& ws) {
    return reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(ws.data_ptr()) + 255) & ~(uintptr_t)255);
}

// A checkpoint in Python: (storage, codes address, exponents address, rows,
// cols, code stride, exponent stride)
py::tuple pack_tuple(const at::Tensor& buf, const iso_act& a) {
    return py::make_tuple(buf, reinterpret_cast<uintptr_t>(a.codes), reinterpret_cast<uintptr_t>(a.exps), a.rows,
                          a.cols, a.ld_codes, a.ld_exps);
}
at::Tensor new_pack(int64_t rows, int64_t cols, const at::Tensor& like, iso_act& a) {
    const int64_t groups = (cols + ISO_ACT_GROUP - 1) / ISO_ACT_GROUP, ldc = groups * ISO_ACT_GROUP,
                  lde = (groups + 7) / 8 * 8;
    at::Tensor buf = at::empty({rows * (ldc + lde)}, like.options().dtype(at::kByte));
    char* at = static_cast<char*>(buf.data_ptr());
    a = {at, at + rows * ldc, rows, cols, ldc, lde};
    return buf;
}
iso_act pack_of(const py::tuple& t, at::Tensor& buf) {
    buf = t[0].cast<at::Tensor>();
    return {reinterpret_cast<void*>(t[1].cast<uintptr_t>()), reinterpret_cast<void*>(t[2].cast<uintptr_t>()),
            t[3].cast<int64_t>(), t[4].cast<int64_t>(), t[5].cast<int64_t>(), t[6].cast<int64_t>()};
}
at::ScalarType dtype_of(const py::object& dtype, at::ScalarType otherwise) {
    if (dtype.is_none()) return otherwise;
    if (!THPDtype_Check(dtype.ptr())) type_error("dtype must be a torch.dtype");
    return reinterpret_cast<THPDtype*>(dtype.ptr())->scalar_type;
}

// every function: its result, or the status code of a refusal
py::object act_pack(const at::Tensor& x) {
    const iso_mat m = mat(x, "x");
    void* s = stream_of(x);
    iso_act a;
    const at::Tensor buf = new_pack(m.rows, m.cols, x, a);
    const int32_t rc = iso_act_pack(&m, &a, s);
    return rc ? py::object(py::int_(rc)) : pack_tuple(buf, a);
}

py::object act_unpack(const py::tuple& pack, const py::object& dtype) {
    at::Tensor buf;
    const iso_act a = pack_of(pack, buf);
    const at::ScalarType t = dtype_of(dtype, at::kBFloat16);
    code_of(t, "out");
    void* s = stream_of(buf);
    const at::Tensor out = empty(a.rows, a.cols, t, buf);
    const iso_mat o = new_mat(out);
    const int32_t rc = iso_act_unpack(&a, &o, s);
    return rc ? py::object(py::int_(rc)) : py::cast(out);
}

py::object act_wgrad(const at::Tensor& dy, const py::tuple& pack, const py::object& dtype) {
    const iso_mat d = mat(dy, "dy");
    at::Tensor buf;
    const iso_act a = pack_of(pack, buf);
    const at::ScalarType t = dtype_of(dtype, at::kFloat);
    code_of(t, "out");
    void* s = stream_of(dy);
    same_device(dy, buf);
    const at::Tensor out = empty(d.cols, a.cols, t, dy);
    const iso_mat o = new_mat(out);
    size_t bytes = 0;
    int32_t rc = iso_act_wgrad_workspace_size(&d, &a, &o, &bytes);
    if (!rc) {
        const at::Tensor ws = scratch(bytes, dy);
        rc = iso_act_wgrad(&d, &a, &o, 0, aligned(ws), bytes, nullptr, s);
    }
    return rc ? py::object(py::int_(rc)) : py::cast(out);
}

py::object swiglu_pack(const at::Tensor& gate, const at::Tensor& up) {
    const iso_mat g = mat(gate, "gate"), u = mat(up, "up");
    void* s = stream_of(gate);
    same_device(gate, up);
    const at::Tensor h = empty(g.rows, g.cols, gate.scalar_type(), gate);
    const iso_mat o = new_mat(h);
    iso_act ga, ua;
    const at::Tensor gb = new_pack(g.rows, g.cols, gate, ga), ub = new_pack(g.rows, g.cols, gate, ua);
    const int32_t rc = iso_swiglu_pack(&g, &u, &o, &ga, &ua, s);
    return rc ? py::object(py::int_(rc)) : py::make_tuple(h, pack_tuple(gb, ga), pack_tuple(ub, ua));
}

py::object swiglu_grad(const at::Tensor& dh, const py::tuple& gate, const py::tuple& up, bool need_h) {
    const iso_mat d = mat(dh, "dh");
    at::Tensor gb, ub;
    const iso_act ga = pack_of(gate, gb), ua = pack_of(up, ub);
    void* s = stream_of(dh);
    same_device(dh, gb);
    same_device(dh, ub);
    const at::ScalarType t = dh.scalar_type();
    const at::Tensor dg = empty(d.rows, d.cols, t, dh), du = empty(d.rows, d.cols, t, dh);
    const iso_mat g = new_mat(dg), u = new_mat(du);
    at::Tensor h;
    iso_mat hm{};
    if (need_h) {
        h = empty(d.rows, d.cols, t, dh);
        hm = new_mat(h);
    }
    const int32_t rc = iso_swiglu_grad(&d, &ga, &ua, &g, &u, need_h ? &hm : nullptr, s);
    if (rc) return py::int_(rc);
    return py::make_tuple(dg, du, need_h ? py::cast(h) : py::object(py::none()));
}

void check_ids(const at::Tensor& ids) {
    if (ids.scalar_type() != at::kInt && ids.scalar_type() != at::kLong)
        type_error("ids must be an int32 or int64 tensor");
    if (!ids.is_cuda() || !ids.is_contiguous()) value_error("ids must be a contiguous CUDA tensor");
}

py::object embed(const at::Tensor& table, const at::Tensor& ids, double scale, int64_t pad_id, const py::object& dtype) {
    const iso_mat t = mat(table, "table");
    check_ids(ids);
    const at::ScalarType ot = dtype_of(dtype, table.scalar_type());
    code_of(ot, "out");
    void* s = stream_of(table);
    same_device(table, ids);
    const at::Tensor out = empty(ids.numel(), t.cols, ot, table);
    const iso_mat o = new_mat(out);
    const int32_t rc = iso_embed(&t, ids.data_ptr(), ids.scalar_type() == at::kLong, ids.numel(), pad_id, (float)scale,
                                 &o, nullptr, s);
    return rc ? py::object(py::int_(rc)) : py::cast(out);
}

py::object embed_grad(const at::Tensor& dy, const at::Tensor& ids, int64_t rows, double scale, int64_t pad_id,
                      const py::object& dtype) {
    const iso_mat d = mat(dy, "dy");
    check_ids(ids);
    if (ids.numel() != d.rows)
        value_error(std::to_string(ids.numel()) + " ids for " + std::to_string(d.rows) + " rows of dy");
    if (rows < 0) value_error("rows must not be negative");
    const at::ScalarType t = dtype_of(dtype, at::kFloat);
    code_of(t, "out");
    void* s = stream_of(dy);
    same_device(dy, ids);
    const at::Tensor out = empty(rows, d.cols, t, dy);
    const iso_mat o = new_mat(out);
    size_t bytes = 0;
    int32_t rc = iso_embed_grad_workspace_size(d.rows, d.cols, &bytes);
    if (!rc) {
        const at::Tensor ws = scratch(bytes, dy);
        rc = iso_embed_grad(&d, ids.data_ptr(), ids.scalar_type() == at::kLong, pad_id, (float)scale, &o, 0, aligned(ws),
                            bytes, nullptr, s);
    }
    return rc ? py::object(py::int_(rc)) : py::cast(out);
}

}  // namespace

PYBIND11_MODULE(_iso_train, m) {
    m.def("act_pack", &act_pack);
    m.def("act_unpack", &act_unpack);
    m.def("act_wgrad", &act_wgrad);
    m.def("swiglu_pack", &swiglu_pack);
    m.def("swiglu_grad", &swiglu_grad);
    m.def("embed", &embed);
    m.def("embed_grad", &embed_grad);
}
