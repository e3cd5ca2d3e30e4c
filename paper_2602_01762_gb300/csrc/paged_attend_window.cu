// The paged attention (paged_attend.cu) over a sliding window and a few first rows.
//
// Row j of L is seen where j < sinks or j >= L - window.  The blocks of 64 rows without
// a seen row are not part of the work that is split, so that the cost goes by the
// window, not by the sequence: rows that are not seen are not read, and neither are the
// block-table entries of pages without a seen row, whose pages can be given back.  The
// weights of a cache that has them are another kernel's, which still counts through all
// blocks of the sequences and passes over those that are not seen.
// Measured, 16 sequences of 1000 to 65536 rows, 8 KV heads of 128 and 4 query heads each,
// a window of 1024 and 4 sinks, bf16: 15.7 us (67 MB, 4.3 TB/s; 4.6 us to the first rows);
// with weights 12 us more, 13 where every sequence has 65536 rows.
#include "paged_attend_tiles.cuh"

namespace prism {

cudaError_t prepare_window_attend_kernels(bool bf16, int D, int G) { return prepare_attend_tiles<WindowRows>(bf16, D, G); }

cudaError_t start_window_attend(const AttendArgs &a, bool bf16, int D, int ht, int sms, cudaStream_t s) {
    return start_attend_tiles<WindowRows>(a, bf16, D, ht, sms, s);
}

cudaError_t prepare_code_attend_kernels(bool bf16, int D, int G) {
    const cudaError_t e = prepare_e4m3_attend(bf16, D, G);
    return e != cudaSuccess ? e : prepare_int8_attend(bf16, D, G);
}

// Codes have one form for both: without a window the window is every row.
cudaError_t launch_code_attend(const CodeAttendArgs &args, CodeFormat format, bool bf16, int D, int sms, cudaStream_t s) {
    CodeAttendArgs a = args;
    if (a.window < 0) a.window = 0x7FFFFFFF;
    a.by_page = Divisor((uint32_t)a.cache.page_size);
    a.by_scale = Divisor((uint32_t)a.scale_rows);
    const PagedView &c = a.cache;
    const long long scales = (long long)a.Hkv * a.scale_blocks, most = 0x7FFFFFFF;
    if (c.page_size % kRunRows == 0 && c.page_stride <= most && c.page_stride >= -most && c.row_stride <= most / 8 && c.row_stride >= -most / 8 &&
        scales * c.n_pages <= most) {
        a.run = c.row_stride == D ? 2 : 1;
        a.short_page = (int)c.page_stride, a.short_row = (int)c.row_stride, a.page_scales = (int)scales;
    }
    return format == kE4m3 ? start_e4m3_attend(a, bf16, D, sms, s) : start_int8_attend(a, bf16, D, sms, s);
}

}  // namespace prism
