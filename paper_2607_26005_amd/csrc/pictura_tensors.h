// What the binding's two native files share: tensors as the library's structs, after
// every check that keeps a kernel inside its buffers.
#pragma once

#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <sstream>
#include <stdexcept>
#include <string>
#include <tuple>
#include <utility>
#include <vector>

#include "pictura_overlap.h"

extern PyMethodDef pictura_calls[];   // pictura_calls.cpp

namespace {

struct Refused : std::runtime_error {
    using std::runtime_error::runtime_error;
};

template <class... A>
[[noreturn]] void refuse(const A&... a)
{
    std::ostringstream s;
    (void)(s << ... << a);
    throw Refused(s.str());
}

int32_t dtype_code(const at::Tensor& t, const char* what)
{
    switch (t.scalar_type()) {
    case at::kFloat: return 0;
    case at::kBFloat16: return 1;
    case at::kHalf: return 2;
    default: refuse(what, ": dtype ", t.scalar_type(), ", expected float32, bfloat16 or float16");
    }
}

// pictura_sequences (include/pictura.h)
struct Sequences {
    uint64_t gates, inputs, state, resets;
    int64_t gates_batch, gates_step, inputs_batch, inputs_step, resets_batch, resets_step, batch, steps;
    int32_t channels, dtype;
};
static_assert(sizeof(Sequences) == 104, "pictura_sequences");

struct Place {
    uint64_t at = 0;
    int64_t batch = 0, step = 0;
};

void strided(const at::Tensor& t, const char* name, const at::Device& dev)
{
    if (t.layout() != at::kStrided || t.is_neg()) refuse(name, ": expected a plain strided tensor");
    if (t.device() != dev) refuse(name, ": tensor on ", t.device(), ", the others are on ", dev);
}

// A tensor [batch, steps, channels] (step: [batch, channels]) whose channels are neighbours.
Place place(const at::Tensor& t, const char* name, const at::Tensor& like, bool whole)
{
    strided(t, name, like.device());
    if (t.scalar_type() != like.scalar_type()) refuse(name, ": dtype ", t.scalar_type(), ", the gates have ", like.scalar_type());
    if (t.sizes() != like.sizes()) refuse(name, ": shape ", t.sizes(), ", the gates have ", like.sizes());
    if (t.size(-1) > 1 && t.stride(-1) != 1) refuse(name, ": strides ", t.strides(), ": a step's channels have to be contiguous");
    return Place{(uint64_t)(uintptr_t)t.data_ptr(), t.stride(0), whole ? t.stride(1) : 0};
}

bool apart(const Sequences& q, const Place& p)
{
    const bool many = q.batch > 1, more = q.steps > 1;
    if ((many && p.batch < q.channels) || (more && p.step < q.channels)) return false;
    return !many || !more || p.batch / p.step >= q.steps || p.step / p.batch >= q.batch;
}

const at::Tensor& given(PyObject* o, const char* name)
{
    if (!THPVariable_Check(o)) refuse(name, ": expected a torch tensor on the HIP device, got ", Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}

const at::Tensor* optional(PyObject* o, const char* name) { return o == Py_None ? nullptr : &given(o, name); }

// Address of a contiguous fp32 tensor [batch, channels], or of the states that a scan saves.
uint64_t floats(const Sequences& q, const at::Tensor& like, const at::Tensor& t, const char* name, bool saved)
{
    constexpr int64_t kSteps = 16;   // PICTURA_SCAN_STEPS
    const int64_t rows = (q.steps + kSteps - 1) / kSteps;
    strided(t, name, like.device());
    if (t.scalar_type() != at::kFloat || t.dim() != (saved ? 3 : 2) || (saved && t.size(0) != rows) || t.size(saved) != q.batch ||
        t.size(saved + 1) != q.channels || !t.is_contiguous())
        refuse(name, ": ", t.scalar_type(), " ", t.sizes(), " with strides ", t.strides(), ", expected contiguous float32 [",
               saved ? std::to_string(rows) + ", " : "", q.batch, ", ", q.channels, "]");
    return (uint64_t)(uintptr_t)t.data_ptr();
}

Sequences sequences_of(bool whole, const at::Tensor& gates, const at::Tensor& inputs, const at::Tensor* state,
                       const at::Tensor* resets)
{
    if (gates.dim() != (whole ? 3 : 2) || gates.size(-1) < 1)
        refuse("gates: shape ", gates.sizes(), ", expected ", whole ? "[batch, steps, channels]" : "[batch, channels]");
    Sequences q{};
    q.dtype = dtype_code(gates, "gates");
    q.batch = gates.size(0);
    q.steps = whole ? gates.size(1) : 1;
    const int64_t channels = gates.size(-1);
    if (channels > 0x7FFFFFFF || q.batch > 0x7FFFFFFF / channels || q.steps > 0x7FFFFFFF)
        refuse("gates: shape ", gates.sizes(), ": batch times channels, and steps, have to be below 2^31");
    q.channels = (int32_t)channels;
    const Place g = place(gates, "gates", gates, whole), x = place(inputs, "inputs", gates, whole);
    q.gates = g.at, q.gates_batch = g.batch, q.gates_step = g.step;
    q.inputs = x.at, q.inputs_batch = x.batch, q.inputs_step = x.step;
    if (state) q.state = floats(q, gates, *state, "state", false);
    if (resets) {
        const at::Tensor& r = *resets;
        strided(r, "resets", gates.device());
        if (r.scalar_type() != at::kBool && r.scalar_type() != at::kByte)
            refuse("resets: dtype ", r.scalar_type(), ", expected bool or uint8");
        if (r.dim() != (whole ? 2 : 1) || r.size(0) != q.batch || (whole && r.size(1) != q.steps))
            refuse("resets: shape ", r.sizes(), ", expected [", q.batch, whole ? ", " + std::to_string(q.steps) : "", "]");
        q.resets = (uint64_t)(uintptr_t)r.data_ptr();
        q.resets_batch = r.stride(0);
        q.resets_step = whole ? r.stride(1) : 0;
    }
    return q;
}

// What a step writes, `out` and the state, may be an operand's own rows and nothing else that is
// read or written.
void check_step(const Sequences& q, int64_t size, const Place& out, uint64_t state)
{
    using namespace pictura;
    auto rows = [&](uint64_t at, int64_t batch) { return region((const void*)at, q.batch, q.channels * size, batch * size); };
    const Region y = rows(out.at, out.batch), h = region((const void*)state, q.batch, q.channels * 4ll, q.channels * 4ll),
                 flags = region((const void*)q.resets, q.batch, 1, q.resets_batch);
    const std::pair<Region, const char*> read[] = {{rows(q.gates, q.gates_batch), "the gates"}, {rows(q.inputs, q.inputs_batch), "the inputs"}};
    for (const auto& [r, name] : read) {
        if (overlap(r, y) && !same(r, y)) refuse("out: overlaps ", name, ", and is not the same rows");
        if (overlap(r, h) && !same(r, h)) refuse("state: overlaps ", name, ", and is not the same rows");
    }
    if (overlap(y, h) && !same(y, h)) refuse("out: overlaps the state, and is not the same rows");
    if (overlap(flags, y)) refuse("out: overlaps the resets");
    if (overlap(flags, h)) refuse("state: overlaps the resets");
}

// pictura_norm (include/pictura.h)
struct Norm {
    uint64_t x, residual, weight;
    int64_t x_stride, residual_stride, rows;
    int32_t width, dtype, weight_dtype;
    float eps;
};
static_assert(sizeof(Norm) == 64, "pictura_norm");

// (address, elements between rows) of a [rows, width] tensor whose rows are contiguous; written: and apart.
std::pair<uint64_t, int64_t> rows_at(const at::Tensor& t, const char* name, const at::Tensor& like, bool written)
{
    strided(t, name, like.device());
    if (t.sizes() != like.sizes()) refuse(name, ": shape ", t.sizes(), ", expected ", like.sizes());
    const int64_t stride = t.size(0) > 1 ? t.stride(0) : t.size(1);
    if ((t.size(1) > 1 && t.stride(1) != 1) || (written && stride < t.size(1)))
        refuse(name, ": strides ", t.strides(), ": a row has to be contiguous", written ? ", and apart from the next" : "");
    return {(uint64_t)(uintptr_t)t.data_ptr(), stride};
}

void same_type(const at::Tensor& t, const char* name, const at::Tensor& x)
{
    if (t.scalar_type() != x.scalar_type()) refuse(name, ": dtype ", t.scalar_type(), ", the others have ", x.scalar_type());
}

Norm norm_of(const at::Tensor& x, const at::Tensor& weight, const at::Tensor* residual, double eps)
{
    constexpr int64_t kMost = 1 << 16;   // PICTURA_MAX_NORM
    Norm q{};
    q.dtype = dtype_code(x, "x");
    if (x.dim() != 2 || x.size(1) < 1 || x.size(1) > kMost || x.size(0) > 0x7FFFFFFF)
        refuse("x: shape ", x.sizes(), ": rows of 1 to ", kMost, " elements, fewer than 2^31 of them");
    q.rows = x.size(0);
    q.width = (int32_t)x.size(1);
    std::tie(q.x, q.x_stride) = rows_at(x, "x", x, false);
    strided(weight, "weight", x.device());
    q.weight_dtype = dtype_code(weight, "weight");
    if (weight.dim() != 1 || weight.size(0) != q.width || !weight.is_contiguous() ||
        (weight.scalar_type() != x.scalar_type() && weight.scalar_type() != at::kFloat))
        refuse("weight: ", weight.scalar_type(), " ", weight.sizes(), " with strides ", weight.strides(), ", expected contiguous ",
               x.scalar_type(), " or float32 [", q.width, "]");
    q.weight = (uint64_t)(uintptr_t)weight.data_ptr();
    if (residual) {
        same_type(*residual, "residual", x);
        std::tie(q.residual, q.residual_stride) = rows_at(*residual, "residual", x, false);
    }
    if (!(eps >= 0) || eps > 3e38) refuse("eps: expected a finite number, 0 or more");
    q.eps = (float)eps;
    return q;
}

}  // namespace
