// Argument checks shared by the C-ABI entry points of the operators on rows.  Each check returns an empty text if all is well.
#pragma once
#include <new>

#include "head.h"

namespace hadfl {
namespace checks {

constexpr int kMaxRows = 1 << 20, kMaxCols = 1 << 17, kMaxClasses = 1 << 20;
constexpr long long kMaxLines = 1ll << 24;

inline hadfl_status bad(const std::string& msg) { return fail_call(HADFL_EINVAL, msg); }

template <typename F> hadfl_status guarded(F&& body) noexcept
{
    try { return body(); }
    catch (const std::bad_alloc&) {
        try { return fail_call(HADFL_ENOMEM, "out of host memory"); } catch (...) { return HADFL_ENOMEM; }
    }
    catch (...) {
        try { return fail_call(HADFL_ENOMEM, "unexpected host exception"); } catch (...) { return HADFL_ENOMEM; }
    }
}

inline hadfl_status done(hipError_t e, const char* what)
{
    return e == hipSuccess ? HADFL_OK : fail_call(HADFL_EDEVICE, std::string(what) + ": " + hipGetErrorString(e));
}

inline std::string check_sizes(int n, int rows, int bf16)
{
    if (n < 1 || n > kMaxReplicas) return "n_replicas must be in [1, 1024]";
    if (rows < 0 || rows > kMaxRows) return "n_rows must be in [0, 2^20]";
    if ((long long)n * rows > kMaxLines) return "n_replicas * n_rows must be at most 2^24";
    if (bf16 != 0 && bf16 != 1) return "bf16 must be 0 or 1";
    return "";
}
inline std::string check_cols(const char* name, int cols, int most = kMaxCols)
{
    if (cols >= 1 && cols <= most) return "";
    return std::string(name) + " must be in [1, " + std::to_string(most) + "]";
}

// A tensor of n x rows x cols elements; rows == 1 for a vector per replica.  Strides are bounded so that no offset in bytes
// leaves 63 bits.
inline std::string check_rows(const char* name, const hadfl_rows* r, int n, int rows, int cols, int bf16, bool out, bool vector = false)
{
    const std::string who = name;
    if (!r) return who + " is null";
    if (n == 0 || rows == 0) return "";
    if (!r->data) return who + " has no data";
    if ((uintptr_t)r->data & (bf16 ? 1 : 3)) return who + " is not aligned to its elements";
    const long long most = 1ll << 40, row = vector ? 0 : r->row_stride;
    if (r->replica_stride < 0 || r->replica_stride > most || row < 0 || row > most) return who + ": strides must be in [0, 2^40]";
    if (!out) return "";
    if (!vector && rows > 1 && row < cols) return who + ": row_stride must be at least the columns of an output";
    if (n > 1 && r->replica_stride < (rows - 1) * row + cols) return who + ": the replicas of an output must not overlap";
    return "";
}
inline std::string check_work(const char* name, const void* p, unsigned align)
{
    if (!p) return std::string(name) + " is null";
    if ((uintptr_t)p & (align - 1)) return std::string(name) + " must be " + std::to_string(align) + "-byte aligned";
    return "";
}

inline std::string first(std::initializer_list<std::string> texts)
{
    for (const std::string& t : texts) if (!t.empty()) return t;
    return "";
}

}  // namespace checks
}  // namespace hadfl
