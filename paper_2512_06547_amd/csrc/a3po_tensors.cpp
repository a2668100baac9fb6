// The binding's look at lists of tensors: what the interpreter asks a tensor for costs 40 ns each time, five times a tensor.
#include <torch/csrc/autograd/python_variable.h>

extern "C" {

// Addresses and sizes of a list's tensors.  All have to be dense tensors on the GPU `device`, contiguous, of the first's dtype and,
// where `want` is given, of these numbers of elements.  Returns how many tensors are right: the list's length if all are.
__attribute__((visibility("default"))) int64_t a3po_tensor_list(PyObject *list, int64_t device, const int64_t *want, int64_t *address, int64_t *size)
{
    const int64_t n = PyList_GET_SIZE(list);
    for (int64_t i = 0; i < n; ++i) {
        PyObject *o = PyList_GET_ITEM(list, i);
        if (!THPVariable_Check(o)) return i;
        try {  // (tensors without memory throw when asked for it)
            const at::Tensor &t = THPVariable_Unpack(o);
            if (t.layout() != at::kStrided || !t.is_cuda() || t.get_device() != device || !t.is_contiguous()) return i;
            if (t.scalar_type() != THPVariable_Unpack(PyList_GET_ITEM(list, 0)).scalar_type()) return i;
            if (want && t.numel() != want[i]) return i;
            address[i] = reinterpret_cast<int64_t>(t.data_ptr());
            if (size) size[i] = t.numel();
        } catch (...) {
            return i;
        }
    }
    return n;
}

}
