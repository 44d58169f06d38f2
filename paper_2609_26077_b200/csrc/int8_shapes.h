// How the 8-bit layer's row kernels are launched: plain C++, so that the rules can be checked without a device.
#pragma once

// Row per block or warp (the norm, row-wise quantization): every thread has vpt groups of eight columns.
//   Two groups of eight columns a thread up to 512 columns, four up to 16384; a warp a row up to 1024.  (Two groups a thread up to 4096
//   columns: 16384 x 4096 bf16 in 98.5 instead of 74.3 us, 8192 x 2048 in 25.2 instead of 21.7.)
struct Int8RowForm {
    int vpt;        // groups of eight columns a thread
    int threads;    // of a row; above 512 the row does not fit registers and is read again for each pass
    bool whole;     // the columns fill every thread, so that nothing has to be tested.  Never of a row without columns.
};
inline Int8RowForm int8_row_form(long long cols)
{
    const long long groups = (cols + 7) / 8;
    Int8RowForm f;
    f.vpt = groups <= 64 ? 2 : 4;
    f.threads = (int)((groups + 32 * f.vpt - 1) / (32 * f.vpt) * 32);
    f.whole = cols > 0 && cols == 8ll * f.vpt * f.threads;
    return f;
}
