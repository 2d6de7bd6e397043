// Tables of the adapter kernels' instances for one type; included by the source file of that type.
#pragma once
#include "adapter_launch.cuh"

namespace cs {

template <class T, int TM, int RP, int V>
AdapterKernel row_instance()
{
    using G = AdGeom<T, TM, RP>;
    return {(const void *)k_adapter<T, TM, RP, V>, G::SMEM, G::CTAS, THREADS};
}

template <class T, int TM, int V>
AdapterKernel row_by_rank(int rank)
{
    // rows that allow no 8-byte access are copied value by value: two sizes of that will do
    if (V > 0 && rank <= 16) return row_instance<T, TM, V ? 16 : 64, V>();
    if (V > 0 && rank <= 32) return row_instance<T, TM, V ? 32 : 64, V>();
    if (rank <= 64) return row_instance<T, TM, 64, V>();
    return row_instance<T, TM, 128, V>();
}

template <class T, int TM>
AdapterKernel row_by_vec(int rank, int vec)
{
    return vec == 16 ? row_by_rank<T, TM, 16>(rank) : vec == 8 ? row_by_rank<T, TM, 8>(rank) : row_by_rank<T, TM, 0>(rank);
}

template <class T>
AdapterKernel row_kernel(const RowShape &s)
{
    return s.tm == 16 ? row_by_vec<T, 16>(s.rank, s.vec) : row_by_vec<T, 64>(s.rank, s.vec);
}

template <class T, int RP, int V>
AdapterKernel wgrad_instance(int &strip)
{
    if constexpr (sizeof(T) == 4) {
        using G = WgGeom32<RP>;
        strip = G::WC;
        return {(const void *)k_adapter_wgrad32<RP, V>, G::SMEM, G::SMEM <= 113 * 1024 ? 2 : 1, THREADS};
    } else {
        using G = WgGeom16<T, RP>;
        strip = G::WC;
        return {(const void *)k_adapter_wgrad16<T, RP, V>, G::SMEM, G::CTAS, G::BLOCK};
    }
}

template <class T, int V>
AdapterKernel wgrad_by_rank(int rank, int &strip)
{
    if (V > 0 && rank <= 16) return wgrad_instance<T, V ? 16 : 64, V>(strip);
    if (V > 0 && rank <= 32) return wgrad_instance<T, V ? 32 : 64, V>(strip);
    if (rank <= 64) return wgrad_instance<T, 64, V>(strip);
    return wgrad_instance<T, 128, V>(strip);
}

template <class T>
AdapterKernel wgrad_kernel(int rank, int vec, int &strip)
{
    return vec == 16 ? wgrad_by_rank<T, 16>(rank, strip) : vec == 8 ? wgrad_by_rank<T, 8>(rank, strip) : wgrad_by_rank<T, 0>(rank, strip);
}

}  // namespace cs
