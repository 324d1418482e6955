// Lists of torch tensors for the Python binding: reading a tensor's address, shape and type takes some tenths of a microsecond each from Python, which for a
// list of hundreds of gradients is longer than the work on them (1000 of them and their outputs: 1690 us, here 12).  Called with the interpreter's lock held
// (ctypes.PyDLL); not part of the C interface.
#include <torch/csrc/autograd/python_variable.h>
#include "../../include/silenzio_clear.h"

static bool type_of(const at::Tensor &t, int &type) {
    switch (t.scalar_type()) {
    case at::kFloat: type = SLZ_F32; return true;
    case at::kBFloat16: type = SLZ_BF16; return true;
    case at::kHalf: type = SLZ_F16; return true;
    default: return false;
    }
}

// The table of gradients and outputs, two lists of the same length: 0, or 1 where a tensor is not a plain one (contiguous, of a type that is taken, on `device`, without a gradient
// of its own where `recording`, at most 2^31 - 1 elements, its output of the same shape and type): the caller then looks at them one by one, and says what is wrong.
extern "C" int slz_tensors_table(PyObject *grads, PyObject *outputs, int device, int recording, slz_grad_tensor *table) {
    try {
        if (!PyList_Check(grads) || !PyList_Check(outputs) || PyList_GET_SIZE(grads) != PyList_GET_SIZE(outputs)) return 1;
        for (Py_ssize_t i = 0; i < PyList_GET_SIZE(grads); i++) {
            PyObject *po = PyList_GET_ITEM(outputs, i), *pg = PyList_GET_ITEM(grads, i);
            if (!THPVariable_Check(pg) || !THPVariable_Check(po)) return 1;
            const at::Tensor &g = THPVariable_Unpack(pg), &o = THPVariable_Unpack(po);
            int type, type_o;
            for (const at::Tensor *t : {&g, &o})
                if (!t->is_cuda() || t->get_device() != device || !t->is_contiguous() || t->numel() > 0x7fffffff || (recording && t->requires_grad())) return 1;
            if (!type_of(g, type) || !type_of(o, type_o) || type != type_o || g.sizes() != o.sizes()) return 1;
            const uint32_t n = (uint32_t)g.numel();
            table[i] = {g.data_ptr(), o.data_ptr(), 1u, n, n, n, type};
        }
        return 0;
    } catch (...) {
        return 1;
    }
}
// The list's tensors have been written to: backward passes that kept one of them notice
extern "C" int slz_tensors_written(PyObject *tensors) {
    try {
        for (Py_ssize_t i = 0; i < PyList_GET_SIZE(tensors); i++) {
            const at::Tensor &t = THPVariable_Unpack(PyList_GET_ITEM(tensors, i));
            if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
        }
        return 0;
    } catch (...) {
        return 1;
    }
}
