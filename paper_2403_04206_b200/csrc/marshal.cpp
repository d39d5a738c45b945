// Pointer tables of the replica operators for the Python binding: checks the tensors of a call and writes
// their addresses into host arrays, in one call from Python (attribute by attribute in Python, the checks of
// a call with 24 tensors take longer than its launch).  Marshalling only; no tensor is created or changed.  The arrays
// are bytes objects that belong to the call (ctypes passes their address): between this module's checks and the C
// call Python may run anything, another call with other tables included.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <Python.h>

#include <cstdint>
#include <memory>
#include <string>

namespace {

constexpr int kMaxWorkers = 64, kMaxTables = 12;

// A reference that is given back on every way out (questions to a tensor may throw).
struct GiveBack { void operator()(PyObject* o) const { Py_DECREF(o); } };
using Ref = std::unique_ptr<PyObject, GiveBack>;

enum Mode { kRows = 1, kOptional = 2, kFloat32 = 4 };

bool fail(PyObject* type, const char* name, const std::string& text)
{
    PyErr_SetString(type, (std::string(name) + ": " + text).c_str());
    return false;
}

// One table: (name, tensors or None, rows, cols, mode).  mode kRows: 2-D tensors [rows, cols] whose rows may be
// padded, all with one row stride; else contiguous tensors of rows * cols elements, whose stride is given as 0: matrices
// [rows, cols] (a transposed one has as many elements, in another order), or, where cols is 1 or the tensor is no
// matrix, any that hold as many.  Below the stride, in the lowest 4 bits of *layout: the bits below 16 that any of the
// addresses has.  *table: bytes, or the integer 0 for None.
bool one_table(PyObject* spec, Py_ssize_t workers, at::ScalarType kind, int device, PyObject** table, int64_t* layout)
{
    const char* name;
    PyObject* bufs;
    long long rows, cols;
    int mode;
    if (!PyArg_ParseTuple(spec, "sOLLi", &name, &bufs, &rows, &cols, &mode)) return false;
    int64_t stride = (mode & kRows) ? cols : 0, low = 0;
    *layout = stride << 4;
    if (bufs == Py_None) {
        if (!(mode & kOptional)) return fail(PyExc_TypeError, name, "expected a list of tensors, got None");
        *table = PyLong_FromLong(0);
        return *table != nullptr;
    }
    const Ref held(PySequence_Fast(bufs, "expected a list of tensors"));
    PyObject* const list = held.get();
    if (list == nullptr) return false;
    bool ok = true;
    uint64_t address[kMaxWorkers];
    if (PySequence_Fast_GET_SIZE(list) != workers)
        ok = fail(PyExc_ValueError, name, "one entry per worker is needed (" + std::to_string(workers) + "), got " + std::to_string(PySequence_Fast_GET_SIZE(list)));
    if (mode & kFloat32) kind = at::kFloat;
    for (Py_ssize_t m = 0; ok && m < workers; ++m) {
        PyObject* item = PySequence_Fast_GET_ITEM(list, m);
        if (!THPVariable_Check(item)) { ok = fail(PyExc_TypeError, name, "expected tensors"); break; }
        const at::Tensor& t = THPVariable_Unpack(item);
        if (t.scalar_type() != kind) { ok = fail(PyExc_TypeError, name, std::string("expected ") + c10::toString(kind) + ", got " + c10::toString(t.scalar_type())); break; }
        if (!t.is_cuda() || t.get_device() != device) {
            ok = fail(PyExc_ValueError, name, "expected tensors on the current CUDA device (" + std::to_string(device) + "), got " + t.device().str());
            break;
        }
        if (mode & kRows) {
            if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols) {
                ok = fail(PyExc_ValueError, name, "expected shape [" + std::to_string(rows) + ", " + std::to_string(cols) + "]");
                break;
            }
            if (cols > 1 && t.stride(1) != 1) { ok = fail(PyExc_ValueError, name, "the elements of a row must be contiguous"); break; }
            if (rows > 1) {                                   // of a single row the stride says nothing
                if (m > 0 && t.stride(0) != stride) { ok = fail(PyExc_ValueError, name, "all workers need one row stride"); break; }
                stride = t.stride(0);
            }
        } else if (t.numel() != rows * cols || !t.is_contiguous()) {
            ok = fail(PyExc_ValueError, name, "expected contiguous tensors of " + std::to_string(rows * cols) + " elements");
            break;
        }
        if (!(mode & kRows) && t.dim() == 2 && t.size(0) > 1 && t.size(1) > 1 && cols > 1 && (t.size(0) != rows || t.size(1) != cols)) {
            ok = fail(PyExc_ValueError, name, "expected shape [" + std::to_string(rows) + ", " + std::to_string(cols) + "]");
            break;
        }
        address[m] = reinterpret_cast<uint64_t>(t.data_ptr());
        low |= static_cast<int64_t>(address[m] & 15);
    }
    if (!ok) return false;
    *layout = stride << 4 | low;
    *table = PyBytes_FromStringAndSize(reinterpret_cast<const char*>(address), static_cast<Py_ssize_t>(workers * sizeof(uint64_t)));
    return *table != nullptr;
}

// tables(first, device, specs): the storage type code of `first` (a list of tensors, one a worker) and, for each
// spec, its pointer table (bytes; 0 for None) and its layout, 16 * row stride + the low bits of its addresses.
PyObject* tables(PyObject*, PyObject* args)
{
    PyObject *first, *specs;
    int device;
    if (!PyArg_ParseTuple(args, "OiO!", &first, &device, &PyTuple_Type, &specs)) return nullptr;
    try {
        const Py_ssize_t workers = PySequence_Size(first), count = PyTuple_GET_SIZE(specs);
        if (workers < 0) return nullptr;
        if (workers < 1 || workers > kMaxWorkers || count > kMaxTables) {
            PyErr_Format(PyExc_ValueError, "1 to %d workers are possible, got %zd", kMaxWorkers, workers);
            return nullptr;
        }
        const Ref item(PySequence_GetItem(first, 0));
        if (item == nullptr) return nullptr;
        const bool tensor = THPVariable_Check(item.get());
        const at::ScalarType kind = tensor ? THPVariable_Unpack(item.get()).scalar_type() : at::kByte;
        const int code = kind == at::kFloat ? 0 : kind == at::kBFloat16 ? 1 : kind == at::kHalf ? 2 : -1;
        if (code < 0) {
            PyErr_SetString(PyExc_TypeError, "expected CUDA tensors of float32, bfloat16 or float16");
            return nullptr;
        }
        Ref result(PyTuple_New(1 + 2 * count));
        PyObject* const out = result.get();
        if (out == nullptr) return nullptr;
        PyTuple_SET_ITEM(out, 0, PyLong_FromLong(code));
        for (Py_ssize_t i = 0; i < count; ++i) {
            PyObject* table = nullptr;
            int64_t layout = 0;
            if (!one_table(PyTuple_GET_ITEM(specs, i), workers, kind, device, &table, &layout)) return nullptr;
            PyTuple_SET_ITEM(out, 1 + 2 * i, table);
            PyTuple_SET_ITEM(out, 2 + 2 * i, PyLong_FromLongLong(layout));
        }
        return result.release();
    } catch (python_error& e) {                               // raised by a tensor's own Python code
        e.restore();
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

PyMethodDef methods[] = {{"tables", tables, METH_VARARGS, "Checked pointer tables of a replica operator's tensors."}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
