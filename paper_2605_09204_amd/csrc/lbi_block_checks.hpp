// What the C entry points of the region blocks' operators check of their arguments, and how they
// lay out a workspace (host code).
#ifndef LBI_BLOCK_CHECKS_HPP
#define LBI_BLOCK_CHECKS_HPP

#include <initializer_list>

#include "lbi_block_internal.h"

namespace lbi {
namespace {

constexpr int64_t kMostRows = (int64_t)1 << 40;  // of a token or state tensor
constexpr int64_t kMostValues = (int64_t)1 << 46;

inline size_t size_of(lbi_dtype dt) { return dt == LBI_F32 ? 4 : 2; }
inline bool known(lbi_dtype dt) { return dt == LBI_F32 || dt == LBI_BF16; }

// A tensor of `rows` rows of `cols` elements at a stride of `ld`; data may be
// NULL where it is optional.
struct Tensor {
    const void *data;
    int64_t rows, cols, ld;
    size_t element;
    size_t bytes() const
    {
        return data && rows > 0 && cols > 0 ? ((size_t)(rows - 1) * ld + cols) * element : 0;
    }
};
inline Tensor tokens(const void *p, int64_t rows, int64_t cols, int64_t ld, size_t element)
{
    return {p, rows, cols, ld, element};
}
inline Tensor dense(const void *p, int64_t rows, int64_t cols, size_t element)
{
    return {p, rows, cols, cols, element};
}
inline bool overlap(const Tensor &a, const Tensor &b)
{
    const uintptr_t pa = (uintptr_t)a.data, pb = (uintptr_t)b.data;
    const size_t na = a.bytes(), nb = b.bytes();
    if (!(na && nb && pa < pb + nb && pb < pa + na))
        return false;
    const size_t stride = a.ld * a.element;
    if (stride != b.ld * b.element)
        return true;
    // slices of the rows of one buffer: apart where their columns are
    const size_t ca = a.cols * a.element, cb = b.cols * b.element;
    const size_t ab = pb >= pa ? (pb - pa) % stride : (stride - (pa - pb) % stride) % stride;
    return ab < ca || ab + cb > stride;
}
inline bool same(const Tensor &a, const Tensor &b)
{
    return a.data == b.data && a.rows == b.rows && a.ld == b.ld && a.cols == b.cols &&
           a.element == b.element;
}

// Strides, alignment of elements, and that no output overlaps anything else,
// except `inplace` (an output) and `over` (an input) where they are the same.
inline lbi_status check_tensors(std::initializer_list<Tensor> inputs, std::initializer_list<Tensor> outputs,
                         const Tensor *inplace = nullptr, const Tensor *over = nullptr)
{
    for (const auto *list : {&inputs, &outputs})
        for (const Tensor &t : *list) {
            if (!t.data)
                continue;
            if (t.ld < t.cols || t.rows > kMostRows || (t.rows && t.ld > kMostValues / t.rows))
                return LBI_ERR_SHAPE;
            if ((uintptr_t)t.data & (t.element - 1))
                return LBI_ERR_ALIGN;
        }
    for (const Tensor *o = outputs.begin(); o != outputs.end(); ++o) {
        for (const Tensor *p = outputs.begin(); p != o; ++p)
            if (overlap(*o, *p))
                return LBI_ERR_ALIAS;
        for (const Tensor &i : inputs) {
            if (!overlap(*o, i))
                continue;
            if (!(inplace && over && o->data == inplace->data && i.data == over->data &&
                  same(*o, i)))
                return LBI_ERR_ALIAS;
        }
    }
    return LBI_OK;
}

inline lbi_status check_workspace(const void *workspace, size_t bytes, size_t need)
{
    if (need == 0)
        return LBI_OK;
    if (!workspace || bytes < need)
        return LBI_ERR_WORKSPACE;
    return (uintptr_t)workspace & 255u ? LBI_ERR_ALIGN : LBI_OK;
}

inline lbi_status status_of(hipError_t e) { return e == hipSuccess ? LBI_OK : LBI_ERR_HIP; }

// Lays arrays out in a workspace, 256 bytes apart.
struct Layout {
    char *base;
    size_t used = 0;
    template <typename T> T *take(int64_t count)
    {
        T *p = base ? (T *)(base + used) : nullptr;
        used += ((size_t)count * sizeof(T) + 255) / 256 * 256;
        return p;
    }
};

inline bool bad_norm_shape(int64_t T, int32_t D, float eps)
{
    return T < 0 || T > kMostRows || D < 1 || D > LBI_NORM_MAX_D || !(eps >= 0.f);
}

}  // namespace
}  // namespace lbi

#endif  // LBI_BLOCK_CHECKS_HPP
