// Calls of the operators for language models without a GPU: this program stands in for the HIP runtime (its definitions come before those of the shared
// library), so that the C entry points run their host code and launches are printed.  Addresses are numbers that nothing follows.
//   lm_calls_driver libnetmax.so < calls
// A call is a line: linear, grad, orth, policy or preference, then name=number for members of its shape struct and its arguments; what is not named is 0.
// The line "kernels" is answered by all kernels of the library.
// work=ADDRESS comes with the size that the call's workspace function gives.  A line of output: status, '|', text of the error, '|', launches as
// name<template arguments>@workgroups, without spaces.
#include <hip/hip_runtime_api.h>

#include <cstdio>
#include <cstdlib>
#include <cxxabi.h>
#include <dlfcn.h>
#include <iostream>
#include <map>
#include <sstream>
#include <string>

#include "../include/netmax.h"

static std::map<const void *, std::string> g_names;
static dim3 g_grid, g_block;
static size_t g_shared;
static hipStream_t g_stream;
static std::ostringstream g_out;

// "void netmax::name<...>(...)" as name<...>; 16-bit types that the demangler may not know by names that it does
static std::string plain_name(std::string mangled)
{
    for (const auto &[from, to] : {std::pair<std::string, std::string>("DF16b", "u6__bf16"), {"DF16_", "Dh"}})
        for (size_t at; (at = mangled.find(from)) != std::string::npos;) mangled.replace(at, from.size(), to);
    int status = 0;
    char *whole = abi::__cxa_demangle(mangled.c_str(), nullptr, nullptr, &status);
    const std::string s(whole ? whole : mangled);
    free(whole);
    const size_t from = s.find("netmax::");
    std::string of;
    int depth = 0;
    for (size_t k = from == std::string::npos ? 0 : from + 8; k < s.size() && (depth > 0 || s[k] != '('); ++k) {
        depth += s[k] == '<' ? 1 : s[k] == '>' ? -1 : 0;
        if (s[k] != ' ') of += s[k];
    }
    return of;
}

extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *handle; return &handle; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
void __hipRegisterFunction(void **, const void *function, char *, const char *name, unsigned, void *, void *, dim3 *, dim3 *, int *) { g_names[function] = plain_name(name); }
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t shared, hipStream_t s)
{
    g_grid = grid; g_block = block; g_shared = shared; g_stream = s;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *shared, hipStream_t *s)
{
    *grid = g_grid; *block = g_block; *shared = g_shared; *s = g_stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *function, dim3 grid, dim3, void **, size_t, hipStream_t)
{
    g_out << ' ' << g_names[function] << '@' << (uint64_t)grid.x * grid.y * grid.z;
    return hipSuccess;
}
const char *hipGetErrorString(hipError_t) { return "error"; }
hipError_t hipGetLastError() { return hipSuccess; }
}

int main(int argc, char **argv)
{
    void *lib = argc == 2 ? dlopen(argv[1], RTLD_NOW) : nullptr;
    if (!lib) {
        fprintf(stderr, "%s\n", argc == 2 ? dlerror() : "usage: lm_calls_driver libnetmax.so < calls");
        return 2;
    }
#define ENTRY(name) const auto name##_ = reinterpret_cast<decltype(&name)>(dlsym(lib, #name))
    ENTRY(netmax_linear); ENTRY(netmax_linear_workspace); ENTRY(netmax_linear_grad); ENTRY(netmax_linear_grad_workspace); ENTRY(netmax_orthogonalize);
    ENTRY(netmax_orthogonalize_workspace); ENTRY(netmax_policy_loss); ENTRY(netmax_preference_loss); ENTRY(netmax_preference_workspace); ENTRY(netmax_last_error);
#undef ENTRY
    for (std::string line; std::getline(std::cin, line);) {
        std::istringstream in(line);
        std::string op;
        in >> op;
        std::map<std::string, double> v;                            // addresses stay below 2^53
        for (std::string word; in >> word;) v[word.substr(0, word.find('='))] = std::stod(word.substr(word.find('=') + 1));
        const auto n = [&](const char *name) { return (int64_t)v[name]; };
        const auto f = [&](const char *name) { return (float)v[name]; };
        const auto p = [&](const char *name) { return reinterpret_cast<float *>((uintptr_t)v[name]); };
        const auto i = [&](const char *name) { return reinterpret_cast<int32_t *>((uintptr_t)v[name]); };
        g_out.str("");
        int rc = -100;
        if (op == "kernels")
            for (const auto &k : g_names) g_out << ' ' << k.second << "@0";
        if (op == "linear" || op == "grad") {
            const netmax_linear_shape s{n("batch"), n("rows"), n("d_in"), n("d_out"), (int32_t)n("dtype"), (int32_t)n("act"), n("ldx"), n("ldw"), n("ldr"), n("ldy"), n("ldz"), n("sx"), n("sw"),
                                        n("sb"), n("sr"), n("sy"), n("sz"), n("lddx"), n("lddw"), n("sdx"), n("sdw"), n("sdb")};
            if (op == "linear")
                rc = netmax_linear_(&s, p("x"), p("w"), p("bias"), p("residual"), p("y"), p("z"), p("work"), netmax_linear_workspace_(&s, p("x"), p("w")), nullptr);
            else
                rc = netmax_linear_grad_(&s, p("dy"), p("x"), p("w"), p("z"), p("dx"), p("dw"), p("db"), p("work"), netmax_linear_grad_workspace_(&s, p("dy"), p("x"), p("w")), nullptr);
        } else if (op == "orth") {
            const netmax_orth_shape s{n("batch"), n("rows"), n("cols"), (int32_t)n("dtype"), (int32_t)n("steps"), (int32_t)n("nesterov"), f("mu"), f("a"), f("b"), f("c"), f("eps"), f("scale"),
                                      n("ldg"), n("sg"), n("ldm"), n("sm"), n("ldo"), n("so")};
            rc = netmax_orthogonalize_(&s, p("g"), p("m"), p("m_out"), p("out"), p("work"), netmax_orthogonalize_workspace_(&s), nullptr);
        } else if (op == "policy") {
            rc = netmax_policy_loss_(n("tokens"), n("vocab"), (int32_t)n("dtype"), p("logits"), n("ld"), i("labels"), p("old_logp"), p("ref_logp"), p("advantage"), p("weight"), f("low"), f("high"),
                                     f("kl"), p("loss"), p("logp"), p("grad"), n("ldg"), nullptr);
        } else if (op == "preference") {
            rc = netmax_preference_loss_(n("tokens"), n("vocab"), (int32_t)n("dtype"), p("logits"), n("ld"), i("labels"), n("pairs"), i("offsets"), p("ref_logp"), p("weight"), f("beta"),
                                         f("smoothing"), f("scale"), p("loss"), p("ratio"), p("grad"), n("ldg"), p("work"), netmax_preference_workspace_(n("tokens"), n("pairs")), nullptr);
        }
        printf("%d|%s|%s\n", rc, rc == NETMAX_OK ? "" : netmax_last_error_(nullptr), g_out.str().c_str());
    }
    return 0;
}
