// What binding.py does once per tensor argument and once per call, without the interpreter: checks and the address of a tensor, and torch's current stream.
//   ptr(tensor or None, dtype or None) -> address or None; the checks and errors of binding._ptr_any, which serves everything that is not a plain tensor
//   stream() -> the current stream of the current device
//   quantized_cache(k, v, k_scale, v_scale) -> (pages, kv heads, page size, head dimension, type, addresses of the four) of an 8-bit cache
//   kv_rows(k, v, kv heads, head dimension) -> (rows, stride between rows, addresses of the two) of K/V rows
//   (both: AssertionError where the tensors are not what the call takes; in Python these checks were half of a small call's time)
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

PyObject* g_any = nullptr;                            // binding._ptr_any

PyObject* ptr(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n < 1 || n > 2) {
        PyErr_SetString(PyExc_TypeError, "ptr(tensor, dtype=None)");
        return nullptr;
    }
    PyObject* t = args[0];
    PyObject* dtype = n == 2 ? args[1] : Py_None;
    if (t == Py_None) Py_RETURN_NONE;
    if (THPVariable_CheckExact(t) && (dtype == Py_None || THPDtype_Check(dtype))) {
        const at::Tensor& x = THPVariable_Unpack(t);
        if (x.is_cuda() && x.is_contiguous() && (dtype == Py_None || x.scalar_type() == reinterpret_cast<THPDtype*>(dtype)->scalar_type))
            return PyLong_FromVoidPtr(x.data_ptr());
    }
    return PyObject_CallFunctionObjArgs(g_any, t, dtype, nullptr);
    END_HANDLE_TH_ERRORS
}

PyObject* stream(PyObject*, PyObject*)
{
    HANDLE_TH_ERRORS
    return PyLong_FromVoidPtr(c10::hip::getCurrentHIPStream().stream());
    END_HANDLE_TH_ERRORS
}

const at::Tensor* tensor(PyObject* t) { return THPVariable_Check(t) ? &THPVariable_Unpack(t) : nullptr; }

PyObject* refuse(const char* why)
{
    PyErr_SetString(PyExc_AssertionError, why);
    return nullptr;
}

PyObject* quantized_cache(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor* x[4];
    if (n != 4) return refuse("quantized_cache(k_cache, v_cache, k_scale, v_scale)");
    for (int i = 0; i < 4; ++i)
        if (!(x[i] = tensor(args[i])) || !x[i]->is_cuda() || !x[i]->is_contiguous()) return refuse("an 8-bit cache and its scales: device-resident contiguous tensors only");
    const auto type = x[0]->scalar_type();
    if ((type != at::kFloat8_e4m3fn && type != at::kChar) || x[1]->scalar_type() != type) return refuse("an 8-bit cache: float8_e4m3fn or int8, K and V alike");
    if (x[0]->dim() != 4 || x[1]->sizes() != x[0]->sizes()) return refuse("an 8-bit cache: [pages, kv heads, page size, head dimension], K and V alike");
    for (int i = 2; i < 4; ++i)
        if (x[i]->scalar_type() != at::kFloat || x[i]->dim() != 2 || x[i]->size(0) != x[0]->size(0) || x[i]->size(1) != x[0]->size(1))
            return refuse("scales of an 8-bit cache: float32 [pages, kv heads]");
    return Py_BuildValue("LLLLiNNNN", (long long)x[0]->size(0), (long long)x[0]->size(1), (long long)x[0]->size(2), (long long)x[0]->size(3), type == at::kChar ? 1 : 0,
                         PyLong_FromVoidPtr(x[0]->data_ptr()), PyLong_FromVoidPtr(x[1]->data_ptr()), PyLong_FromVoidPtr(x[2]->data_ptr()), PyLong_FromVoidPtr(x[3]->data_ptr()));
    END_HANDLE_TH_ERRORS
}

PyObject* kv_rows(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 4) return refuse("kv_rows(k, v, Hkv, D)");
    const int64_t Hkv = PyLong_AsLongLong(args[2]), D = PyLong_AsLongLong(args[3]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor* x[2] = {tensor(args[0]), tensor(args[1])};
    int64_t stride = 0;
    for (int i = 0; i < 2; ++i) {
        if (!x[i] || !x[i]->is_cuda() || x[i]->scalar_type() != at::kBFloat16) return refuse("K/V rows: device-resident bfloat16 tensors only");
        if (x[i]->dim() != 3 || x[i]->size(0) != x[0]->size(0) || x[i]->size(1) != Hkv || x[i]->size(2) != D) return refuse("K/V rows: [rows, kv heads, head dimension] of the cache");
        // (where there is one row, one head or one element, the stride says nothing)
        if ((D > 1 && x[i]->stride(2) != 1) || (Hkv > 1 && x[i]->stride(1) != D)) return refuse("K/V rows: contiguous inside a row only");
        const int64_t between = x[i]->size(0) > 1 ? x[i]->stride(0) : Hkv * D;
        if (i && between != stride) return refuse("K/V rows: K and V equally strided");
        stride = between;
    }
    return Py_BuildValue("LLNN", (long long)x[0]->size(0), (long long)stride, PyLong_FromVoidPtr(x[0]->data_ptr()), PyLong_FromVoidPtr(x[1]->data_ptr()));
    END_HANDLE_TH_ERRORS
}

PyObject* set_any(PyObject*, PyObject* f)
{
    Py_INCREF(f);
    Py_XSETREF(g_any, f);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"ptr", (PyCFunction)(void (*)(void))ptr, METH_FASTCALL, nullptr},
                         {"quantized_cache", (PyCFunction)(void (*)(void))quantized_cache, METH_FASTCALL, nullptr},
                         {"kv_rows", (PyCFunction)(void (*)(void))kv_rows, METH_FASTCALL, nullptr},
                         {"stream", stream, METH_NOARGS, nullptr},
                         {"set_any", set_any, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
