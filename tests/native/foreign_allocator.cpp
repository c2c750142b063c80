// Tensors on the GPU whose memory comes from an allocator of its own, for the test of where results come from.  Called through ctypes with the interpreter's lock held.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <ATen/EmptyTensor.h>
#include <c10/core/Allocator.h>

namespace {

struct Foreign final : c10::Allocator {
    long long calls = 0;
    c10::DataPtr allocate(size_t n) override
    {
        ++calls;
        return at::empty({0}, at::device(at::kCUDA)).storage().allocator()->allocate(n);
    }
    c10::DeleterFnPtr raw_deleter() const override { return nullptr; }
    void copy_data(void *, const void *, size_t) const override { TORCH_CHECK(false, "nothing is copied"); }
} foreign;

}  // namespace

extern "C" PyObject *foreign_float_tensor(long long rows, long long columns)
{
    const int64_t shape[] = {rows, columns};
    return THPVariable_Wrap(at::Tensor(at::detail::empty_generic(shape, &foreign, c10::DispatchKeySet(c10::DispatchKey::CUDA), at::kFloat, std::nullopt)));
}
extern "C" long long foreign_calls() { return foreign.calls; }
