// Where the kernels around a language model's layers work, by the arguments of their launches: lm_step_calls_driver.cpp, which sees each launch's arguments as well.
// Behind a launch that would do something wrong comes what, in the form of a launch: name@amount.
//   behind_the_workspace@bytes   a kernel's last row of partial sums, of means or of unwanted results ends so far behind the part of the workspace that it was given
//   sums_of_no_rows@n            n partial sums are joined that no row has left
//   clears_kept_rows@workgroups  so many workgroups of a gradient of an embedding that accumulates would clear rows
//   clears_behind_the_table@row  a workgroup would clear rows from there on, which the table does not have
#include <hip/hip_runtime.h>
#define hipLaunchKernel lm_calls_launch
#include "lm_step_calls_driver.cpp"
#undef hipLaunchKernel

#include "../paper_2009_05766_amd/csrc/block_norm.h"
#include "../paper_2009_05766_amd/csrc/embed.h"

#include <algorithm>

using namespace netmax;

static void wrong(const char *what, int64_t amount)
{
    if (amount > 0) g_out << ' ' << what << '@' << amount;
}

// The template argument number k of a kernel's name.
static std::string argument(const std::string &name, int k)
{
    size_t at = name.find('<') + 1;
    for (; k > 0; --k) at = name.find(',', at) + 1;
    return name.substr(at, name.find_first_of(",>", at) - at);
}

static void look_at_norm(const std::string &name, dim3 grid, dim3 block, void **args)
{
    const NormArgs &a = *(const NormArgs *)args[0];
    const Partials &to = *(const Partials *)args[1];
    const char *const start = (const char *)to.p, *const end = start + to.bytes, *const rows = to.rows ? (const char *)to.rows : (const char *)to.unwanted;
    const int64_t partials = 4 * a.batch * to.workgroups * to.sums * to.padded;
    wrong("behind_the_workspace", start + partials - rows);
    if (to.rows) wrong("behind_the_workspace", (const char *)(to.rows + a.batch * a.rows) - (const char *)to.unwanted);
    if (name.rfind("join_sums_kernel<", 0) == 0 && a.rows == 0) wrong("sums_of_no_rows", to.workgroups);
    if (name.rfind("norm_grad_kernel<", 0) != 0) return;
    const int64_t groups = block.x / std::stoi(argument(name, 1));
    const bool block_form = argument(name, 4) != "0", gated = argument(name, 4) >= "3";
    if (a.dx.p && (!block_form || a.df.p) && (!gated || a.dgate.p)) return;
    const int64_t last = to.unwanted_row(grid.y - 1, grid.x - 1, groups - 1, groups);
    wrong("behind_the_workspace", (const char *)to.unwanted + (last + a.width) * (a.bf16 ? 2 : 4) - end);
}

static void look_at_embed(const EmbedArgs &a, const GradTurns &turns, dim3 grid, int64_t rows_to_clear)
{
    int64_t kept = 0, behind = 0;
    for (int64_t id = turns.sums; id < (int64_t)grid.x * grid.y; ++id) {
        if (!turns.clears((uint32_t)id)) continue;
        kept += a.accumulate;
        if ((id - turns.sums) * rows_to_clear >= a.vocab) behind = std::max(behind, (id - turns.sums) * rows_to_clear);
    }
    wrong("clears_kept_rows", kept);
    wrong("clears_behind_the_table", behind);
}

extern "C" hipError_t hipLaunchKernel(const void *function, dim3 grid, dim3 block, void **args, size_t shared, hipStream_t s)
{
    const hipError_t launched = lm_calls_launch(function, grid, block, args, shared, s);
    const std::string &name = g_names[function];
    if (name.rfind("norm_grad_kernel<", 0) == 0 || name.rfind("norm_columns_kernel<", 0) == 0 || name.rfind("long_norm_grad_kernel<", 0) == 0 || name.rfind("join_sums_kernel<", 0) == 0)
        look_at_norm(name, grid, block, args);
    const EmbedArgs *a = (const EmbedArgs *)args[0];
    if (name.rfind("embed_grad_narrow_kernel<", 0) == 0) look_at_embed(*a, *(const GradTurns *)args[1], grid, *(const int *)args[2]);
    if (name.rfind("embed_grad_few_kernel<", 0) == 0) look_at_embed(*a, *(const GradTurns *)args[2], grid, *(const int *)args[3]);
    if (name.rfind("embed_sum_kernel<", 0) == 0) look_at_embed(*a, *(const GradTurns *)args[3], grid, 64);
    return launched;
}
