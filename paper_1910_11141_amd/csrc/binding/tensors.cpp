// What a table of tensors holds of each: read from the tensors of a Python list at once, for calls over some hundred of them (learning.py).  Asked one by
// one from Python each of five attributes takes 50 to 100 ns.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>
#include <exception>
#include <utility>
#include <vector>

namespace {

// NUTS_F32, NUTS_BF16, NUTS_F16 of nuts.h, or -1
int64_t type_of(const at::Tensor& t)
{
    switch (t.scalar_type()) {
        case at::ScalarType::Float: return 0;
        case at::ScalarType::BFloat16: return 2;
        case at::ScalarType::Half: return 3;
        default: return -1;
    }
}

// Stretches of memory, n of them in kept[0], each from kept[1 + 2 k] up to kept[2 + 2 k], apart and in order.  Tensors of a list mostly lie in an order, too: the
// gap between two stretches that one lies in is where the next is looked for first.
struct Kept {
    const int64_t* kept;
    int64_t n, gap = 0;  // the gap in front of stretch `gap`
    explicit Kept(const int64_t* k) : kept(k), n(k ? k[0] : 0) {}
    int64_t begin(int64_t k) const { return kept[1 + 2 * k]; }
    int64_t end(int64_t k) const { return kept[2 + 2 * k]; }
    bool meets(int64_t from, int64_t to)
    {
        if (n == 0 || from >= to) return false;
        if ((gap > 0 && end(gap - 1) > from) || (gap < n && end(gap) <= from)) {
            int64_t low = 0, high = n;  // the first that ends behind `from`
            while (low < high) {
                const int64_t middle = (low + high) / 2;
                if (end(middle) > from) high = middle;
                else low = middle + 1;
            }
            gap = low;
        }
        return gap < n && begin(gap) < to;
    }
};

}  // namespace

// Tensors are read as this PyTorch's headers lay them out: who loads this library looks for the mark first.
extern "C" __attribute__((visibility("default"), used)) const char nuts_reader_mark[] = NUTS_READER_MARK;

// For each item i of `list` (of a tensor, or None), of its address, count and type those into rows[i * width + column] whose column is not negative (0 and
// nothing for None).  Returns bits: 1 tensors of several types, 2 on several devices, 4 with gaps, 8 of another shape than the item of `like` (a list, or
// None) in the same place, 16 an address or a count is not what was in its place, 32 memory of what `kept` (see Kept, or NULL) says.  -1 with an exception: an
// item is neither.
extern "C" __attribute__((visibility("default"))) int nuts_tensor_table(PyObject* list, PyObject* like, int64_t* rows, int64_t width, int64_t address, int64_t count,
                                                                        int64_t type, const int64_t* kept)
try {
    if (!PyList_Check(list) || (like != Py_None && (!PyList_Check(like) || PyList_GET_SIZE(like) != PyList_GET_SIZE(list)))) {
        PyErr_SetString(PyExc_TypeError, "lists of tensors of one length are wanted");
        return -1;
    }
    int bits = 0;
    const at::Tensor* first = nullptr;
    Kept written(kept);
    for (Py_ssize_t i = 0; i < PyList_GET_SIZE(list); ++i) {
        PyObject* item = PyList_GET_ITEM(list, i);
        int64_t* row = rows + i * width;
        if (item == Py_None) {
            if (address >= 0 && row[address] != 0) bits |= 16;
            if (address >= 0) row[address] = 0;
            if (count >= 0 && row[count] != 0) bits |= 16;
            if (count >= 0) row[count] = 0;
            continue;
        }
        if (!THPVariable_Check(item)) {
            PyErr_SetString(PyExc_TypeError, "a tensor is wanted");
            return -1;
        }
        const at::Tensor& t = THPVariable_Unpack(item);
        if (!t.has_storage() || t.layout() != at::kStrided) {
            PyErr_SetString(PyExc_TypeError, "a tensor with memory of its own is wanted");
            return -1;
        }
        if (!first) first = &t;
        if (t.scalar_type() != first->scalar_type()) bits |= 1;
        if (t.device() != first->device()) bits |= 2;
        if (!t.is_contiguous()) bits |= 4;
        if (like != Py_None) {
            PyObject* other = PyList_GET_ITEM(like, i);
            if (!THPVariable_Check(other) || THPVariable_Unpack(other).sizes() != t.sizes()) bits |= 8;
        }
        if (address >= 0) {
            const int64_t at = reinterpret_cast<int64_t>(t.const_data_ptr());
            if (row[address] != at) bits |= 16;
            row[address] = at;
            if (written.meets(at, at + t.numel() * (int64_t)t.element_size())) bits |= 32;
        }
        if (count >= 0) {
            if (row[count] != t.numel()) bits |= 16;
            row[count] = t.numel();
        }
        if (type >= 0) row[type] = type_of(t);
    }
    return bits;
} catch (const std::exception& e) {  // (tensors of kinds that have no memory to ask for)
    PyErr_SetString(PyExc_TypeError, e.what());
    return -1;
}

// Of the tensors without gaps of two lists (or None in their place), of those bits 1 and 2, and 64 where any two overlap.  -1 with an exception: an item is no
// tensor.
extern "C" __attribute__((visibility("default"))) int nuts_tensors_compare(PyObject* one, PyObject* other)
try {
    int bits = 0;
    const at::Tensor* first = nullptr;
    std::vector<std::pair<int64_t, int64_t>> spans;
    for (PyObject* list : {one, other}) {
        if (!PyList_Check(list)) {
            PyErr_SetString(PyExc_TypeError, "lists of tensors are wanted");
            return -1;
        }
        spans.reserve(spans.size() + PyList_GET_SIZE(list));
        for (Py_ssize_t i = 0; i < PyList_GET_SIZE(list); ++i) {
            PyObject* item = PyList_GET_ITEM(list, i);
            if (item == Py_None) continue;
            if (!THPVariable_Check(item)) {
                PyErr_SetString(PyExc_TypeError, "a tensor is wanted");
                return -1;
            }
            const at::Tensor& t = THPVariable_Unpack(item);
            if (!first) first = &t;
            if (t.scalar_type() != first->scalar_type()) bits |= 1;
            if (t.device() != first->device()) bits |= 2;
            const int64_t at = reinterpret_cast<int64_t>(t.const_data_ptr());
            if (t.numel() > 0) spans.emplace_back(at, at + t.numel() * (int64_t)t.element_size());
        }
    }
    if (!std::is_sorted(spans.begin(), spans.end())) std::sort(spans.begin(), spans.end());
    for (size_t k = 1; k < spans.size(); ++k)
        if (spans[k - 1].second > spans[k].first) bits |= 64;
    return bits;
} catch (const std::exception& e) {
    PyErr_SetString(PyExc_TypeError, e.what());
    return -1;
}
