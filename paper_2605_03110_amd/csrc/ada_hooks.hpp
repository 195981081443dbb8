// What the library's translation units share on the host (ada_kernels.hip has it).
#pragma once
#include <hip/hip_runtime.h>

#define ADA_HIDDEN __attribute__((visibility("hidden")))

ADA_HIDDEN void* ada_hook_prof_open(int cls, hipStream_t st);   // a kernel's launch begins / has been made (ada_profile_enable)
ADA_HIDDEN void ada_hook_prof_close(void* scope);
ADA_HIDDEN int ada_hook_cus();                                  // compute units, whole XCDs

struct ProfHook {
    void* scope;
    ProfHook(int cls, hipStream_t st) : scope(ada_hook_prof_open(cls, st)) {}
    ~ProfHook() { ada_hook_prof_close(scope); }
    ProfHook(const ProfHook&) = delete;
    ProfHook& operator=(const ProfHook&) = delete;
};

template <int N> struct Const { static constexpr int value = N; };
