// The loads of every tile that the 8-bit kernels are made of, by the list that they are made from (f8_loader.hpp), as emu_f8_loads.cpp checks them.
#define main main_of_loads
#include "emu_f8_loads.cpp"
#undef main

#include "../../paper_2406_10707_amd/csrc/f8_forms.hpp"

namespace {

template <int FORM>
void products() {
    if constexpr (FORM < kF8FormCount) {
        typedef typename F8GemmShape<FORM>::type S;
        if (S::BM != int(kF8Forms[FORM].bm) || S::BN != int(kF8Forms[FORM].bn)) fail("not the table's tile");
        tiles<S>(kF8Forms[FORM].name);
        products<FORM + 1>();
    }
}

}  // namespace

int main() {
    products<0>();
    tiles<F8GatedShape<0>::type>("gated, 256 tokens");
    tiles<F8GatedShape<1>::type>("gated, 128 tokens");
    tiles<F8GatedShape<2>::type>("gated, 64 tokens");
    tiles<F8GatedValuesShape>("gated, values first");
    tiles<F8BackwardShape>("gated, backward");
    printf("ok %llu loads\n", count);
}
