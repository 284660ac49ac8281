// fp32 to an output type, to nearest even.
#pragma once

namespace {

template <typename T> __device__ __forceinline__ T narrow(float v) { return (T)v; }
// The compiler makes one instruction of a product and its rounding to fp16, which rounds once where fp32 outputs and bf16 round twice.  All
// types are to get the same fp32 value, so the product is kept apart from the rounding.
template <> __device__ __forceinline__ _Float16 narrow<_Float16>(float v)
{
    asm("" : "+v"(v));
    return (_Float16)v;
}

}  // namespace
