// Launches of kernels on rows that waves hold in registers (rows_device.h), by a plan (rows_plan.h).
#pragma once
#include "anr_kernels.h"
#include "element_types.h"
#include "rows_plan.h"

namespace anr {
namespace rows {

template <typename T>
constexpr int values_of(int64_t C) { return C >= 16 / (int)sizeof(T) ? 16 / (int)sizeof(T) : 1; }

// f(V, U, WHOLE) as constants for rows of C elements T, by a plan.
template <typename T, typename F>
hipError_t with_rows(int64_t C, const Plan& p, F f)
{
    constexpr int V = 16 / (int)sizeof(T);
    if (C < V) return f(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{}, std::true_type{});
    auto of = [&](auto u) { return C % V == 0 ? f(std::integral_constant<int, V>{}, u, std::true_type{}) : f(std::integral_constant<int, V>{}, u, std::false_type{}); };
    switch (p.units) {
        case 1: return of(std::integral_constant<int, 1>{});
        case 2: return of(std::integral_constant<int, 2>{});
        case 4: return of(std::integral_constant<int, 4>{});
        default:
            if constexpr (V == 4) return of(std::integral_constant<int, 8>{});
            else return of(std::integral_constant<int, 4>{});
    }
}

template <typename T>
Plan plan_for(int64_t C, int64_t T_)
{
    const int V = values_of<T>(C);
    return plan_of((C + V - 1) / V, kHeld / V, T_);
}

template <typename T>
BackwardPlan backward_plan_for(int64_t C, int64_t T_)
{
    const int V = values_of<T>(C);
    return backward_plan_of((C + V - 1) / V, kHeld / V, T_);
}

}  // namespace rows
}  // namespace anr
